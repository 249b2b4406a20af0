// What the forms of attention over a paged cache share: the list of work, how it is cut over the CTAs, which positions a
// row sees, and how the pieces of a unit are left for the kernel that joins them.
//
// A unit is RU query rows (row = token * share + head of the group) of one sequence and key head; its work is the tiles of
// KT positions that some of its rows see (the first tokens' tiles, then those from the window's start on).  The tiles of all units,
// with an entry cost for each unit's start, form one list that is cut into equal pieces, one per CTA, whatever the lengths
// are: a CTA meets at most two units that it shares with others, its first and its last.  Lengths are known on the device only,
// so every CTA works the list out for itself (a lane per sequence or, where they are many, per row tile, and a scan; about 1.5 us of latency).  It reads
// packing and lengths once and keeps them in shared memory: all its warps go by the same numbers, and come to their ends by them, also where
// somebody changes the arrays under a call.
#pragma once

#include "paged.cuh"

namespace coreinfer {

constexpr float kLog2e = 1.4426950408889634f;

// Which CTAs work on a unit that is cut; written by the CTA that has its first tile, read by the joining kernel.
struct PagedPiece {
    int b, h, tile;         // sequence, key head, row tile
    int last;               // the last CTA with a piece of it; below 0: nothing to join
};

struct PagedAttnArgs {
    Paged c;
    const uint8_t* q;
    uint8_t* out;
    long long ld_q, ld_out;
    int share;              // query heads per key head, and what divides by it:
    unsigned share_mul, share_shift;
    int window, sinks;      // window 0: everything before a token
    float scale2;           // scale * log2(e)
    int RU, KT, cost;       // rows of a unit, positions of a tile (powers of two), entries that a unit's start counts
    int ru_shift, kt_shift; // log2 of the two
    int n_ctas;
    unsigned* status;       // the workspace's first word
    PagedPiece* pieces;     // [n_ctas]
    float2* part_ml;        // [n_ctas][2][RU]: reference exponent (base 2) and sum
    float* part_o;          // [n_ctas][2][D / 4][RU][4]: rows side by side, as the threads that write them are
};

// The tensor-core form (paged_attention_tc.cu): 16-bit caches.
static inline int paged_chunk_rows(int head_dim) { return head_dim == 256 ? 128 : 256; }
constexpr int kPagedChunkTile = 128;
constexpr int kPagedChunkCtas = 148;
coreinfer_status paged_chunk(PagedAttnArgs& a, bool f16, const DeviceInfo& di, cudaStream_t st);

// The form for few rows (paged_attention_few.cu): 16-bit caches; rows of a unit 8 or 16.
struct PagedFewShape {
    int RU, KT, ctas;
};
static inline PagedFewShape paged_few_shape(int head_dim, int rows) { return {rows <= 8 ? 8 : 16, head_dim == 64 ? 256 : 128, head_dim * (rows <= 8 ? 1 : 2) >= 256 ? 148 : 296}; }
coreinfer_status paged_few(const PagedAttnArgs& a, bool f16, const DeviceInfo& di, cudaStream_t st);

// n / share = (n * mul) >> 32 >> shift for 0 <= n < 2^31, with mul = ceil(2^(31 + l) / share), l = ceil(log2 share), shift = l - 1: the
// error n (mul share - 2^(31 + l)) / (share 2^(31 + l)) is below 1 / share.  mul 0: share is 1.
static inline void paged_set_share(PagedAttnArgs& a, int share)
{
    a.share = share;
    a.share_mul = a.share_shift = 0;
    if (share == 1) return;
    int l = 1;
    while ((1 << l) < share) ++l;
    a.share_mul = (unsigned)(((1ull << (31 + l)) + share - 1) / share);
    a.share_shift = l - 1;
}

// The form for few rows of fp32 caches (paged_attention_rows.cu): up to four rows a unit.
constexpr int kPagedRowsMost = 4;
static inline int paged_rows_tile(int head_dim) { return 8192 / head_dim; }
coreinfer_status paged_rows_f32(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st);

// Shared memory of the list: its starts [B + 1], then what the sequences are [B].
static inline size_t paged_list_bytes(int B) { return (size_t)(B + 1) * 4 + (size_t)B * 12; }

#ifdef __CUDACC__

static_assert(sizeof(PagedSeq) == 12, "three numbers");
__device__ __forceinline__ PagedSeq* paged_kept(const PagedAttnArgs& a, int* at) { return reinterpret_cast<PagedSeq*>(at + a.c.B + 1); }
__device__ __forceinline__ const PagedSeq& paged_kept(const PagedAttnArgs& a, const int* at, int b) { return reinterpret_cast<const PagedSeq*>(at + a.c.B + 1)[b]; }

__device__ __forceinline__ int by_share(const PagedAttnArgs& a, int n) { return a.share_mul ? (int)(__umulhi((unsigned)n, a.share_mul) >> a.share_shift) : n; }

// The tiles that the rows of a unit see.
struct PagedTiles {
    int count;              // tiles of the unit
    int first_tiles;        // of them, in front: tiles of the first tokens
    int from;               // tile that follows those
    int hi;                 // positions below this are seen by some row
};
__device__ __forceinline__ int paged_rows(const PagedAttnArgs& a, const PagedSeq& s) { return s.n * a.share; }
__device__ __forceinline__ int paged_row_tiles(const PagedAttnArgs& a, const PagedSeq& s) { return (paged_rows(a, s) + a.RU - 1) >> a.ru_shift; }
__device__ __forceinline__ PagedTiles paged_tiles(const PagedAttnArgs& a, const PagedSeq& s, int tile)
{
    const int rows = paged_rows(a, s), r0 = tile * a.RU;
    const int r1 = (r0 + a.RU < rows ? r0 + a.RU : rows) - 1;
    const int p0 = s.position + by_share(a, r0), p1 = s.position + by_share(a, r1);
    PagedTiles t;
    t.hi = clamp_int(p1 + 1, 0, a.c.cap);
    const int lo = a.window ? clamp_int(p0 - a.window + 1, 0, t.hi) : 0;
    t.from = lo >> a.kt_shift;
    const int first = a.sinks < t.hi ? a.sinks : t.hi;
    t.first_tiles = (first + a.KT - 1) >> a.kt_shift;
    if (t.first_tiles > t.from) t.first_tiles = t.from;
    t.count = ((t.hi + a.KT - 1) >> a.kt_shift) - t.from + t.first_tiles;
    return t;
}
__device__ __forceinline__ int paged_tile_at(const PagedTiles& t, int i) { return i < t.first_tiles ? i : i - t.first_tiles + t.from; }

// What one row sees: positions below hi that are at lo or behind it, or below `sinks`.
struct PagedRow {
    int lo, hi;
};
__device__ __forceinline__ PagedRow paged_row(const PagedAttnArgs& a, const PagedSeq& s, int row)
{
    const int p = s.position + by_share(a, row);
    PagedRow r;
    r.hi = clamp_int(p + 1, 0, a.c.cap);
    r.lo = a.window ? p - a.window + 1 : 0;
    return r;
}
// Whether it sees anything: a token that lies a window or more behind the table sees the first tokens at most.
__device__ __forceinline__ bool paged_sees_some(const PagedAttnArgs& a, const PagedRow& r) { return r.hi > 0 && (r.lo < r.hi || a.sinks > 0); }
__device__ __forceinline__ bool paged_sees(const PagedAttnArgs& a, const PagedRow& r, int j) { return j < r.hi && (j >= r.lo || j < a.sinks); }

// The list (the host has seen to it that it is shorter than 2^31).  `at`: paged_list_bytes() of shared memory; called by all threads of the
// CTA (a multiple of 32).
__device__ __forceinline__ int paged_plan(const PagedAttnArgs& a, int* at)
{
    const int lane = threadIdx.x & 31;
    for (int b0 = (int)(threadIdx.x >> 5) * 32; b0 < a.c.B; b0 += blockDim.x) {
        // a lane per sequence, and the warp together for those of many row tiles
        const int b = b0 + lane;
        PagedSeq s = {0, 0, 0};
        if (b < a.c.B) paged_kept(a, at)[b] = s = paged_seq(a.c, b);
        const int tiles = paged_row_tiles(a, s);
        int w = 0;
        if (tiles <= 2)
            for (int i = 0; i < tiles; ++i) w += a.cost + paged_tiles(a, s, i).count;
        for (unsigned many = __ballot_sync(0xffffffffu, tiles > 2); many; many &= many - 1) {
            const int l = __ffs(many) - 1;
            const PagedSeq one = {0, __shfl_sync(0xffffffffu, s.n, l), __shfl_sync(0xffffffffu, s.position, l)};
            const int n = __shfl_sync(0xffffffffu, tiles, l);
            int sum = 0;
            for (int i = lane; i < n; i += 32) sum += a.cost + paged_tiles(a, one, i).count;
            sum = __reduce_add_sync(0xffffffffu, sum);
            if (lane == l) w = sum;
        }
        if (b < a.c.B) at[b + 1] = w * a.c.H;
    }
    if (threadIdx.x == 0) at[0] = 0;
    __syncthreads();
    if (threadIdx.x < 32) {
        long long carry = 0;
        for (int b0 = 0; b0 < a.c.B; b0 += 32) {
            const int b = b0 + threadIdx.x;
            long long w = b < a.c.B ? at[b + 1] : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long left = __shfl_up_sync(0xffffffffu, w, d);
                if (threadIdx.x >= d) w += left;
            }
            w += carry;
            if (b < a.c.B) at[b + 1] = (int)w;
            carry = __shfl_sync(0xffffffffu, w, 31);
        }
        // sequences that share rows, as no packing has them, can exceed what the host allowed for: then nothing is done
        if (threadIdx.x == 0 && carry > 0x7fffffff) at[a.c.B] = 0;
    }
    __syncthreads();
    return at[a.c.B];
}
// The list in a piece per CTA, or as many as it has entries: `each` entries, one more in the first `longer` of them.
struct PagedCut {
    int each, longer;
    __device__ __forceinline__ void set(const PagedAttnArgs& a, int total)
    {
        const int n = total < a.n_ctas ? total : a.n_ctas;
        each = (unsigned)total / (unsigned)n;
        longer = total - each * n;
    }
    __device__ __forceinline__ int start(int i) const { return i * each + (i < longer ? i : longer); }
    // The piece that holds entry x.
    __device__ __forceinline__ int owner(int x) const
    {
        const int before = longer * (each + 1);      // at most the list's length
        return x < before ? (unsigned)x / (unsigned)(each + 1) : longer + (unsigned)(x - before) / (unsigned)each;
    }
};

// Walks the units of a piece [x, end) of the list.
struct PagedWalk {
    int x, end;             // entries of the piece not walked yet
    int b, h, tile;
    int base;               // entry where the unit starts
    PagedSeq s;
    PagedTiles t;

    // Called by whole warps.
    __device__ __forceinline__ void begin(const PagedAttnArgs& a, const int* at, int total, int cta)
    {
        x = end = 0;
        if (cta >= total) return;
        PagedCut cut;
        cut.set(a, total);
        x = cut.start(cta);
        end = cut.start(cta + 1);
        int lo = 0, hi = a.c.B;                      // at[lo] <= x < at[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (at[mid] <= x) lo = mid;
            else hi = mid;
        }
        b = lo;
        s = paged_kept(a, at, b);
        const unsigned per_head = (unsigned)(at[b + 1] - at[b]) / (unsigned)a.c.H;
        h = (int)((unsigned)(x - at[b]) / per_head);
        base = at[b] + h * per_head;
        // the row tile, 32 at a time: a lane each
        const int lane = threadIdx.x & 31, tiles = paged_row_tiles(a, s);
        for (tile = 0;; tile += 32) {
            int sum = tile + lane < tiles ? a.cost + paged_tiles(a, s, tile + lane).count : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int left = __shfl_up_sync(0xffffffffu, sum, d);
                if (lane >= d) sum += left;
            }
            const unsigned behind = __ballot_sync(0xffffffffu, base + sum > x);
            if (behind) {
                const int l = __ffs(behind) - 1;
                const int before = __shfl_sync(0xffffffffu, sum, l > 0 ? l - 1 : 0);
                tile += l;
                if (l > 0) base += before;
                break;
            }
            base += __shfl_sync(0xffffffffu, sum, 31);
        }
        t = paged_tiles(a, s, tile);
    }
    __device__ __forceinline__ bool more() const { return x < end; }
    // The last piece that has a part of the unit.  (Worked out again: the registers would be held through every unit.)
    __device__ __forceinline__ int last(const PagedAttnArgs& a, const int* at) const
    {
        PagedCut cut;
        cut.set(a, at[a.c.B]);
        return cut.owner(base + a.cost + t.count - 1);
    }
    // Tiles from .. to - 1 of the unit are this piece's.
    __device__ __forceinline__ int from(const PagedAttnArgs& a) const { return x > base + a.cost ? x - base - a.cost : 0; }
    __device__ __forceinline__ int to(const PagedAttnArgs& a) const
    {
        const int n = end - base - a.cost;
        return n < 0 ? 0 : (n < t.count ? n : t.count);
    }
    __device__ __forceinline__ void next(const PagedAttnArgs& a, const int* at)
    {
        base += a.cost + t.count;
        x = base;
        if (x >= end) return;
        if (++tile == paged_row_tiles(a, s)) {
            tile = 0;
            if (++h == a.c.H) {
                h = 0;
                do ++b; while (at[b + 1] == at[b]);
                s = paged_kept(a, at, b);
            }
        }
        t = paged_tiles(a, s, tile);
    }
};

// What every form leaves for who comes after it, by one thread of a CTA: no unit is cut until one is, and no wait has given up.
__device__ __forceinline__ void paged_first_words(const PagedAttnArgs& a)
{
    a.pieces[blockIdx.x].last = -1;
    if (blockIdx.x == 0) *a.status = kStatusOk;
}
// Rows of a unit.
__device__ __forceinline__ int paged_unit_rows(const PagedAttnArgs& a, const PagedWalk& w)
{
    const int left = paged_rows(a, w.s) - w.tile * a.RU;
    return left < a.RU ? left : a.RU;
}
// The infinities and NaN of one output that a row sees in the piece's tiles that some row of the unit (hi_min, lo_max: of its
// rows) sees in part only.  There they were set to 0 for the product; in the other tiles they reach the sums by themselves.
template <typename T>
__device__ __noinline__ float paged_odd_sum(const PagedAttnArgs& a, const PagedWalk& w, int hi_min, int lo_max, int from, int to, int row, int d)
{
    const PagedRow see = paged_row(a, w.s, row);
    float sum = 0.f;
    for (int i = from; i < to; ++i) {
        const int j0 = paged_tile_at(w.t, i) * a.KT;
        if (j0 + a.KT <= hi_min && (j0 >= lo_max || j0 + a.KT <= a.sinks)) continue;
        for (int j = j0; j < j0 + a.KT; ++j) {
            if (!paged_sees(a, see, j)) continue;
            const int page = paged_page(a.c, w.b, j);
            if (page < 0) continue;
            const float x = to_f32(reinterpret_cast<const T*>(a.c.pool[1])[paged_offset(a.c, page, w.h, j) + d]);
            if (!isfinite(x)) sum += x;
        }
    }
    return sum;
}
// Element offset of a row of a unit in q or out.
__device__ __forceinline__ long long paged_row_offset(const PagedAttnArgs& a, const PagedSeq& s, int h, int row, long long ld)
{
    const int t = by_share(a, row);
    return (long long)(s.first + t) * ld + (long long)(h * a.share + row - t * a.share) * a.c.D;
}

// Whether one of the two 16-bit values is an infinity or NaN.
template <typename T>
__device__ __forceinline__ bool odd_pair(uint32_t w)
{
    constexpr uint32_t E = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
    return (w & E) == E || (w & (E << 16)) == (E << 16);
}
template <typename T>
__device__ __forceinline__ uint32_t without_odd(uint32_t w)
{
    constexpr uint32_t E = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
    if ((w & E) == E) w &= 0xffff0000u;
    if ((w & (E << 16)) == (E << 16)) w &= 0xffffu;
    return w;
}

#endif

}  // namespace coreinfer
