// Attention of a few new tokens per sequence over the 4-bit key/value cache.
//
// Mathematics.  With x^ = s c + o per group, a logit is  sum_g [ s_g sum_{d in g} q_d c_d + o_g sum_{d in g} q_d ]
// and an output  sum_n (p_n s_n) c_nd + sum_n p_n o_n : both products run over the codes themselves, scales enter as factors
// of fp32 sums (keys) or of the fp32 weights p (values).  One pass over the cache with a running maximum per query
// row; rows = new tokens x query heads that share a key head.
// Values average out and codes 0..15 do not: over 130000 slots of equal weight the sum of p s c is some thousand times the
// output, and the MMA's accumulators cut off below their last place.  So every kAttnCentre pieces bf16 calls take 8 times
// what p s came to out of the accumulators, by an MMA with codes that are all -8, and put it into the sum of p o.  An MMA also
// lines its products up by exponent fields, which for a subnormal code is that of 2^-14: what it adds up keeps about
// 2^-18 of the largest product (measured 3 to 5e-6 of the absolute terms).  bf16's one part of p s hides that; fp32 and fp16
// calls subtract 8 from every value code, which makes it a normal number (one more instruction per two codes: 52.7 -> 53.9 us
// at 2 x 8 heads x 4 fp16 rows x 130000 slots, error 4e-8 of the absolute terms).  The sums of q c stay exact with subnormals
// in both, since high parts of q are multiples of one step; fp32 calls start them at -8 sum q.
//
// What bounds it: the bytes of the cache (codes and pairs of keys and values, each read once).  The work per
// byte is what has to be kept small, so the codes go to mma.sync.m16n8k16 as fp16 subnormals (quant4.cuh: one AND
// per two codes), 16 slots on the M side and 8 query rows on the N side: S^T = K Q^T, then O^T = V^T P^T with
// P^T made from the accumulators of S^T by movmatrix.  tcgen05 would leave most of its 128 rows empty, and its
// operands would have to be widened in shared memory first.
//
// kv4_attention_kernel: persistent CTAs of 8 warps.  Each warp walks its own slots, 32 at a time, through a ring of
// stages of its own, each the keys or the values of those slots (cp.async, 16 bytes a lane), and refills a stage as
// soon as it has read it: no warp waits for another before the end of a unit, and a refill costs a dozen
// instructions.  (Bulk copies with barriers cost about 70 per 32 slots: the kernel is bound by instruction issue and
// the ALU pipe before it is bound by memory.)  Warps that hold other rows of the same slots copy for themselves, from L2.
// The tiles of all (sequence, head)
// units form one list, cut into equal pieces, one per CTA, whatever the lengths are; a unit that is cut leaves
// partial results (maximum, sum, output) in the workspace.  kv4_finish_kernel joins those, and turns the
// logits into weights that it adds to the cache's where that is asked for.
// fp32 and fp16 calls carry query rows and p s as two fp16 parts in neighbouring columns (22 bits; four rows per
// tile instead of eight): with one part the rounding of p s (2^-12, times the ratio of s c to the centred
// value, about 3) would exceed fp16's own rounding.  bf16 calls carry one part, which keeps eight rows a tile: some 4e-4 of the
// output, below its rounding to bf16 (against 64 bits 1.7 to 1.8e-3, torch's form in fp32 1.7e-3; the last bit falls the other
// way in a part of the outputs, so the two differ by 1.4e-3).
// Calls of more than eight bf16 rows per key head may take 16 rows per warp (attn_rpt): the codes are unpacked once for two
// MMAs, and values enter as s c + o in fp16 (p itself instead of p s per group), under a power of two per slot that p makes
// up for.  Three roundings of 2^-12, of p, o and the value, below bf16's 2^-9.
// Measured from a graph over two or three sets of inputs, ragged lengths (accumulating but for the last): 8 x 32 heads x up to 4001
// bf16 37.7 us, 3280 GB/s, of which about 16 do not grow with the length (launches, the lists, starting and joining units,
// finishing); up to 16384 slots 104 us, 4870 GB/s, the slope 5800; 6 sequences x 8 heads x 15 rows in groups of 32 x up to
// 9000 slots 48.8 us, bound by instruction issue and latency (640 instructions per 16 slots and warp, 16 warps an SM); 2 x 8
// heads x 4 fp16 rows x up to 130000 slots 53.1 us, 4500 GB/s.  A call on a stream takes 0.5 to 1 us more, the shortest 8.4
// against 7.1.  At the 128 registers of two CTAs per SM some forms spill, 4 to 44 bytes a thread stored (16 rows of head_dim
// 128 in groups of 32: 96; head_dim 256 in groups of 32, of 255 registers: 44 to 72), some ten instructions a piece.
#include "kv4.cuh"

#include <type_traits>

namespace coreinfer {

constexpr int kAttnWarps = 8;
constexpr int kAttnThreads = 32 * kAttnWarps;
// Slots per tile (a piece per warp): pieces of 32, so that waits, votes and addresses are paid once per 32 slots; of 16
// where registers (head_dim 128 in groups of 32) or shared memory (256) do not carry two.
constexpr int kAttnTile16 = 128;
template <int D, int G, int MODE> constexpr int kAttnTile = MODE == 3 ? kAttnTile16 : (D == 256 || (D == 128 && G == 32) ? 128 : 256);
constexpr int kAttnMaxCtas = 320;
constexpr size_t kAttnSmemRoom = 226 * 1024;                 // dynamic shared memory of a CTA on sm_100a, beside 1 KB
constexpr float kNoLogit = -1e30f;
// A unit counts this many tiles more than it has when the list is cut: about what starting it costs a CTA (its query
// rows, the join of its warps).  Measured at 8 sequences x 32 heads x 4096 slots: CTAs with two units ended 3 to 6 us
// after those with one when this was 0.
constexpr int kAttnUnitCost = 2;

struct AttnArgs {
    Kv4 c;
    const void* q;
    void* out;
    long long ld_q, ld_out;
    int T, share;
    int R;                  // query rows per key head: T * share, row r = t * share + head
    int RT;                 // row tiles (of 8 or 4 rows) per CTA, dividing the warps
    int RU;                 // rows per unit: RT * 8 or RT * 4
    int RB;                 // units per (sequence, key head)
    int n_ctas;             // CTAs of the main kernel
    int finish_slots;       // slots per block of the finishing kernel
    float scale;
    int accumulate;
    float2* part_ml;        // [n_ctas][2][RU]: reference exponent and sum of a cut unit's piece
    float* part_o;          // [n_ctas][2][RU][D]
    int2* pieces;           // [B][H][RB]: first and last CTA that works on a unit
    float2* stats;          // [B][H][RB][RU]: the same of whole units, for the weights
    float* logits;          // [B][H][R][cap], base-2 logits; only with accumulate
};

__device__ __forceinline__ int attn_tiles(int len, int tile) { return (len + tile - 1) / tile; }
// Entries of a unit in the list that is cut: kAttnUnitCost without work, then its tiles.
__device__ __forceinline__ int attn_entries(int tiles) { return tiles ? tiles + kAttnUnitCost : 0; }
// The list in n equal pieces, the first `more` of them one longer; every piece has one entry at least.
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

// Two codes c (or 16 c) less 8 (128), as fp16: above 1024 the codes are the low bits of a number whose last place is 1.
// `above` holds 1024 twice in a register: with it as a literal, beside the mask, this takes an instruction more.
__device__ __forceinline__ uint32_t literal_1024()
{
    uint32_t r;
    asm volatile("mov.u32 %0, 0x64006400;" : "=r"(r));
    return r;
}
template <uint32_t MASK>
__device__ __forceinline__ uint32_t centred(uint32_t x, uint32_t above)
{
    static_assert(MASK == 0x000f000fu || MASK == 0x00f000f0u, "even or odd codes");
    uint32_t up;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(up) : "r"(x), "n"(MASK), "r"(above));        // (x & MASK) | above
    const uint32_t middle = MASK == 0x000f000fu ? 0x64086408u : 0x64806480u;
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&up), *reinterpret_cast<const __half2*>(&middle));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }

// A condition that is rarely true and the same for the warp: used as the bound of a loop of at most one round, so that
// the compiler branches around the body instead of executing it under a predicate.
__device__ __forceinline__ int opaque_zero()
{
    int z;
    asm volatile("mov.u32 %0, 0;" : "=r"(z));
    return z;
}

// Pieces of a warp between two centrings (bf16): the accumulators hold at most their sum of p s c off centre, which costs
// about 2^-24 of it per 16 slots: 5e-4 of the output over 130000 slots of equal weight.
constexpr int kAttnCentre = 8;

// Stages of a warp's ring: as many as two CTAs per SM (head_dim 256: one) leave room for.
constexpr int kAttnStages16 = 6;
template <int D, int G, int MODE> constexpr int kAttnStages =
    MODE == 3 ? kAttnStages16 : D == 64 ? 9 : (D == 256 ? (G == 32 ? 6 : 8) : (G == 32 ? (MODE == 0 ? 7 : 9) : (MODE == 0 ? 4 : 5)));

// How far logit + log2 s (base 2) may exceed its running maximum before that is moved.  Rows change their maximum at different
// pieces, and each change rescales all of a warp's outputs: of 15 rows, nearly every piece did (91 of 1100
// instructions a piece).
template <int MODE> constexpr float kAttnRoom = MODE == 3 ? 6.f : 4.f;

// Position in the list of tiles.
struct Cursor {
    int b, hr, tile, nt;
};

// How query rows sit in the 8 columns of an MMA: a row per column; a row per two columns with the second empty
// (up to 4 rows: half the softmax work per lane); a row per two columns, the second for the low part.
// kRows16: two MMAs of eight columns side by side, so that a warp unpacks the codes once for 16 rows.
enum { kRows8 = 0, kRows4 = 1, kRows4Parts = 2, kRows16 = 3 };
// A warp's query rows, and those that the join takes at a time.
template <int MODE> constexpr int kAttnRows = MODE == kRows16 ? 16 : (MODE == kRows8 ? 8 : 4);
template <int MODE> constexpr int kAttnJoinRows = MODE == kRows8 || MODE == kRows16 ? 8 : 4;
// Query rows of kRows16 in shared memory, per row tile of a CTA: fragments of two MMAs, those of the sums over groups, and
// (factor, slots seen) of each row.
template <int D> constexpr int kAttnQueryBytes = 2 * (D / 32) * 512 + 2 * 256 + 16 * 8;

template <typename T, int D, int G, int MODE>
__global__ void __launch_bounds__(kAttnThreads, D <= 128 ? 2 : 1)
kv4_attention_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr bool PARTS = MODE == kRows4Parts, BOTH = MODE == kRows16, WIDE = MODE == kRows4 || PARTS, CENTRED = sizeof(T) == 4;
    // Eight groups and two rows a lane: value pairs are read from shared memory again where they are used, instead of kept over
    // the softmax (160 bytes of spills, 24.3 us at 4 x 8 heads x 8 rows x 4096; so 22.6).
    constexpr bool RELOAD = D / G == 8 && MODE == kRows8;
    constexpr int H32 = D / 32, NG = D / G, RPT = kAttnRows<MODE>, JOIN = kAttnJoinRows<MODE>, TL = RPT / JOIN;
    constexpr int NV = BOTH ? 4 : (WIDE ? 1 : 2);            // query rows whose logits a lane holds: 2 tig + (i & 1) of MMA i >> 1
    constexpr int TILE = kAttnTile<D, G, MODE>;
    constexpr int UN = TILE / (16 * kAttnWarps);             // pieces of 16 slots per step of a warp
    constexpr uint32_t CODE_ROW = D / 2, PAIR_ROW = NG * 4;
    constexpr int CH = 16 * UN;                              // slots of a piece
    constexpr int STAGES = kAttnStages<D, G, MODE>;
    constexpr uint32_t CODES = CH * CODE_ROW, PAIRS = CH * PAIR_ROW, STAGE = CODES + PAIRS;
    static_assert(CODES % 512 == 0 && PAIRS % 16 == 0 && PAIRS <= 512, "copies of 16 bytes a lane");
    const Kv4& c = a.c;

    extern __shared__ __align__(128) uint8_t smem[];
    float* obuf = reinterpret_cast<float*>(smem + (size_t)kAttnWarps * STAGES * STAGE);                // [8 warps][JOIN][D]
    float2* mlbuf = reinterpret_cast<float2*>(obuf + kAttnWarps * JOIN * D);                 // [8 warps][JOIN]
    float2* slot_power = mlbuf + kAttnWarps * JOIN + (BOTH ? warp_number() * 16 : 0);        // kRows16: [8 warps][16] (k, 2^-k)
    uint8_t* queries = reinterpret_cast<uint8_t*>(mlbuf + kAttnWarps * (JOIN + (BOTH ? 16 : 0)));          // [RT][kAttnQueryBytes]
    int* pre = reinterpret_cast<int*>(queries + (BOTH ? a.RT * kAttnQueryBytes<D> : 0));     // [B + 1] entries of a head before sequence b
    int* tiles_before = pre + c.B + 1;                                                       // [B] tiles of a head before sequence b
    int* lens = tiles_before + c.B;                                                          // [B]
    const int tid = threadIdx.x, warp = warp_number(), lane = tid & 31;
    wait_for_stream();       // nothing of an earlier kernel is read or overwritten above
    if (warp == 0) {
        int run = 0, idle = 0;                               // entries, and those without work, so far
        for (int b0 = 0; b0 < c.B; b0 += 32) {
            const int b = b0 + lane;
            const int len = b < c.B ? kv4_length(c, b) : 0;
            const int tiles = attn_tiles(len, TILE), v = attn_entries(tiles);
            int incl = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += u;
            }
            const unsigned used = __ballot_sync(0xffffffffu, tiles > 0);
            if (b < c.B) {
                lens[b] = len;
                pre[b] = run + incl - v;
                tiles_before[b] = pre[b] - idle - __popc(used & ((1u << lane) - 1u)) * kAttnUnitCost;
            }
            idle += __popc(used) * kAttnUnitCost;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) pre[c.B] = run;
    }
    __syncthreads();
    let_next_start();

    const int HR = c.H * a.RB;
    const int total = pre[c.B] * HR;
    const AttnCut cut(a.n_ctas, total);
    const int me = blockIdx.x;
    const int begin = me < cut.n ? cut.start(me) : 0, end = me < cut.n ? cut.start(me + 1) : 0;
    auto token_of = [&](int r) { return a.T == 1 ? 0 : r / a.share; };       // of a query row
    // The unit and tile of entry t of the list; tile < 0: an entry without work before the unit's first tile.
    auto seek = [&](int t) {
        Cursor k;
        int lo = 0, hi = c.B - 1;                            // last b with pre[b] * HR <= t: it has entries
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pre[mid] * HR <= t) lo = mid; else hi = mid - 1;
        }
        k.b = lo;
        k.nt = attn_tiles(lens[lo], TILE);
        const unsigned rem = (unsigned)(t - pre[lo] * HR), per = (unsigned)(k.nt + kAttnUnitCost);
        k.hr = (int)(rem / per);
        k.tile = (int)(rem - k.hr * per) - kAttnUnitCost;
        return k;
    };
    // This CTA's tiles from a cursor on: a tile, then the next one of the unit or the first of the next unit.
    auto advance = [&](Cursor k, int tiles) {
        while (tiles > 0) {
            if (k.tile + tiles < k.nt) {
                k.tile += tiles;
                break;
            }
            tiles -= k.nt - k.tile;
            k.tile = 0;
            if (++k.hr == HR) {
                k.hr = 0;
                do { ++k.b; } while (k.b < c.B && lens[k.b] == 0);
                k.nt = k.b < c.B ? attn_tiles(lens[k.b], TILE) : 0x40000000;
            }
        }
        return k;
    };

    if (begin < end) {
        const int gid = lane >> 2, tig = lane & 3;
        const int rt = warp % a.RT, sg = warp / a.RT, nsg = kAttnWarps / a.RT;
        const int tok0 = (gid >> 1) + (gid & 1) * 4;         // slot of accumulator row gid within 8; row gid + 8: tok0 + 8
        Cursor k = seek(begin);
        // tiles of this CTA: from the first at or after entry `begin` to the last before entry `end`
        auto tile_number = [&](const Cursor& k) { return tiles_before[k.b] * HR + k.hr * k.nt + (k.tile < 0 ? 0 : k.tile); };
        const Cursor z = seek(end - 1);
        const int n_total = tile_number(z) + (z.tile >= 0) - tile_number(k);
        if (k.tile < 0) k.tile = 0;
        uint4 raw[H32][sizeof(T) / 2];                       // query rows of the unit at hand as they are in memory
        auto load_q = [&](const Cursor& k) {
            const int h = a.RB == 1 ? k.hr : k.hr / a.RB, rb = k.hr - h * a.RB;
            const int r = rb * a.RU + rt * RPT + (WIDE ? gid >> 1 : (BOTH ? (sg & 1) * 8 : 0) + gid);
            const int rr = r < a.R && (MODE != kRows4 || (gid & 1) == 0) ? r : 0, rt_ = token_of(rr);
            const T* src = (const T*)a.q + ((long long)k.b * a.T + rt_) * a.ld_q + (long long)(h * a.share + rr - rt_ * a.share) * D + 8 * tig;
#pragma unroll
            for (int j = 0; j < H32; ++j)
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[j][i] = reinterpret_cast<const uint4*>(src + j * 32)[i];
        };
        if (n_total > 0) load_q(k);
        // ---- this warp's ring ----
        const int stride = nsg * CH;
        const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES) * STAGE;
        // Where the copies stand: the segment (the CTA's tiles of one unit) and the warp's next piece in it.
        int f_b = k.b, f_hr = k.hr, f_t = 0, f_n0 = 0, f_end = 0;            // f_t: tiles before the segment's end
        uint32_t f_slot = 0;                                 // 2^32 slots would be more than the GPU holds
        auto feed_open = [&](int tile, int t) {
            for (;;) {
                const int len = lens[f_b], nt = attn_tiles(len, TILE), n = n_total - t < nt - tile ? n_total - t : nt - tile;
                f_t = t + n;
                f_n0 = tile * TILE + sg * CH;
                f_end = (tile + n) * TILE < len ? (tile + n) * TILE : len;
                f_slot = (uint32_t)(f_b * c.H + (a.RB == 1 ? f_hr : f_hr / a.RB)) * (uint32_t)c.cap + (uint32_t)f_n0;
                if (f_n0 < f_end || f_t >= n_total) break;
                tile = 0;
                t = f_t;
                if (++f_hr == HR) {
                    f_hr = 0;
                    do { ++f_b; } while (lens[f_b] == 0);    // there are tiles left, so there is such a sequence
                }
            }
        };
        // Copies the next piece's keys (which = 0) or values to shared address `at`; after the values on to the next piece.
        auto feed = [&](uint32_t at, int which) {
            if (f_n0 < f_end) {
                // whole 16-slot rows: the capacity is a multiple of 16, so they lie within the buffers
                const uint32_t rows = f_end - f_n0 > CH - 16 ? CH : 16;
                const uint8_t* codes = c.codes[which] + (size_t)f_slot * CODE_ROW + lane * 16;
                const uint8_t* pairs = reinterpret_cast<const uint8_t*>(c.pairs[which]) + (size_t)f_slot * PAIR_ROW + lane * 16;
#pragma unroll
                for (uint32_t i = 0; i < CODES; i += 512)
                    if (i < 16 * CODE_ROW) copy16(at + lane * 16 + i, codes + i);
                    else copy16_if(at + lane * 16 + i, codes + i, rows == CH);
                copy16_if(at + CODES + lane * 16, pairs, lane * 16 < rows * PAIR_ROW);
                if (which) {
                    f_n0 += stride;
                    f_slot += stride;
                    if (f_n0 >= f_end && f_t < n_total) {
                        if (++f_hr == HR) {
                            f_hr = 0;
                            do { ++f_b; } while (lens[f_b] == 0);
                        }
                        feed_open(0, f_t);
                    }
                }
            }
            copy_commit();                                   // one group per stage, empty ones too
        };
        if (n_total > 0) {                                   // after the query rows, which would wait behind these copies
            feed_open(k.tile, 0);
#pragma unroll 1
            for (int s = 0; s < STAGES; ++s) feed(ring + s * STAGE, s & 1);
        }
        const uint32_t above = PARTS || BOTH ? literal_1024() : 0u;
        uint32_t stage = 0;                                  // offset of the stage at hand in the ring
        int t = 0;                                           // tiles done
        // Into a step: its stage has arrived, for every lane.  Out of it: all lanes have read it; it takes the piece STAGES
        // steps on.
        auto enter = [&]() {
            copy_wait<STAGES - 1>();
            __syncwarp();
            return smem + (size_t)(warp * STAGES) * STAGE + stage;
        };
        auto leave = [&](int which) {
            __syncwarp();
            feed(ring + stage, STAGES & 1 ? which ^ 1 : which);
            stage = stage + STAGE == STAGES * STAGE ? 0 : stage + STAGE;
        };
        while (t < n_total) {
            const int first_tile = k.tile, b = k.b, len = lens[b], h = a.RB == 1 ? k.hr : k.hr / a.RB, rb = k.hr - h * a.RB;
            const int n_tiles = n_total - t < k.nt - first_tile ? n_total - t : k.nt - first_tile;
            const int row0 = rb * a.RU + rt * RPT;           // first query row of this warp's tile
            if (tid == 0 && first_tile == 0) {
                const int last = pre[b] * HR + k.hr * attn_entries(k.nt) + kAttnUnitCost + k.nt - 1;
                a.pieces[((size_t)b * c.H + h) * a.RB + rb] = make_int2(me, n_tiles == k.nt ? me : cut.owner(last));
            }

            // query rows as the B operand: column gid = row gid (or part gid & 1 of row gid >> 1), 8 values per 32
            uint32_t qf[BOTH ? 1 : H32][4];
            float qsum[BOTH ? 1 : NG][NV], f[BOTH ? 1 : NV];
            int lim[BOTH ? 1 : NV] = {};                     // slots this lane's columns see
            uint8_t* const mine = queries + (BOTH ? rt * kAttnQueryBytes<D> : 0);
            const uint4* const q_frag = reinterpret_cast<const uint4*>(mine) + lane;
            const uint2* const q_sums = reinterpret_cast<const uint2*>(mine + TL * H32 * 512) + lane;
            const float2* const q_row = reinterpret_cast<const float2*>(mine + TL * (H32 * 512 + 256)) + 2 * tig;
            if constexpr (BOTH) {
                // The first two warps of a row tile lay it out, eight rows each: values below 2^6, so that sums over groups
                // are in fp16's range, as two parts.  (bf16 has eight bits: what falls below 2^-24 is 2^-30 of the row.)
                if (sg < 2) {
                    const bool valid = row0 + sg * 8 + gid < a.R;
                    float v[H32][8], m = 0.f, sum[NG];
#pragma unroll
                    for (int g = 0; g < NG; ++g) sum[g] = 0.f;
#pragma unroll
                    for (int j = 0; j < H32; ++j) {
                        unpack8<T>(raw[j], v[j]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (!valid) v[j][e] = 0.f;
                            m = fmaxf(m, fabsf(v[j][e]));
                        }
                    }
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
                    const int x = range_exponent(m);
                    const float up = pow2(6 - x), lo16 = 1.f / 16.f;
#pragma unroll
                    for (int j = 0; j < H32; ++j)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            v[j][e] *= up;
                            sum[j * 32 / G] += v[j][e];
                        }
#pragma unroll
                    for (int j = 0; j < H32; ++j) {
                        const float *p = G == 32 ? &v[j][0] : &v[j & ~1][(j & 1) * 4], *q = G == 32 ? &v[j][4] : &v[j | 1][(j & 1) * 4];
                        reinterpret_cast<uint4*>(mine)[(sg * H32 + j) * 32 + lane] =
                            make_uint4(pack_half2(p[0], q[0]), pack_half2(p[2], q[2]), pack_half2(p[1] * lo16, q[1] * lo16), pack_half2(p[3] * lo16, q[3] * lo16));
                    }
                    float here[2] = {0.f, 0.f};              // sums over groups 2 tig and 2 tig + 1
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
                        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
                        if (tig == g / 2) here[g & 1] = sum[g];
                    }
                    const float h0 = __half2float(__float2half_rn(here[0])), h1 = __half2float(__float2half_rn(here[1]));
                    reinterpret_cast<uint2*>(mine + TL * H32 * 512)[sg * 32 + lane] = make_uint2(pack_half2(h0, h1), pack_half2(here[0] - h0, here[1] - h1));
                    const int rr = row0 + sg * 8 + gid;
                    if (tig == 0)
                        reinterpret_cast<float2*>(mine + TL * (H32 * 512 + 256))[sg * 8 + gid] =
                            make_float2(ldexpf(a.scale * 1.44269504088896341f, x - 6 + 24), __int_as_float(valid ? len - (a.T - 1 - token_of(rr)) : 0));
                }
                __syncthreads();
            } else {
                const bool valid = row0 + (WIDE ? gid >> 1 : gid) < a.R && (MODE != kRows4 || (gid & 1) == 0);
                float v[H32][8], m = 0.f;
#pragma unroll
                for (int j = 0; j < H32; ++j) {
                    unpack8<T>(raw[j], v[j]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (!valid) v[j][e] = 0.f;
                        m = fmaxf(m, fabsf(v[j][e]));
                    }
                }
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
                const int x = range_exponent(m);             // the largest value goes to [2^13, 2^14)
                const float up = pow2(14 - x);
#pragma unroll
                for (int j = 0; j < H32; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[j][e] *= up;
                const int low = PARTS ? gid & 1 : 0;
                const float lo16 = 1.f / 16.f;               // odd codes stand 16 times higher
                // High parts are multiples of 8, fp16's step at the row's largest value, so that their sums are exact (with each value
                // rounded by itself the logits were off by 1.2e-6 of their spread, now by 2e-7).
                auto row_part = [low](float x, float step) { return PARTS ? half_part(x, step, low) : x; };
#pragma unroll
                for (int j = 0; j < H32; ++j) {
                    // the two entries beside each other in step j (code_word)
                    const float *p = G == 32 ? &v[j][0] : &v[j & ~1][(j & 1) * 4], *q = G == 32 ? &v[j][4] : &v[j | 1][(j & 1) * 4];
                    qf[j][0] = pack_half2(row_part(p[0], 8.f), row_part(q[0], 8.f));
                    qf[j][1] = pack_half2(row_part(p[2], 8.f), row_part(q[2], 8.f));
                    qf[j][2] = pack_half2(row_part(p[1] * lo16, .5f), row_part(q[1] * lo16, .5f));
                    qf[j][3] = pack_half2(row_part(p[3] * lo16, .5f), row_part(q[3] * lo16, .5f));
                }
                // The sums of q over a group: the product with codes that are all 1, which carries the 2^-24 of the
                // sums of c q as well.  f undoes both scalings.
                const float ff = ldexpf(a.scale * 1.44269504088896341f, x - 14 + 24);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = g * G / 32; j < (g + 1) * G / 32; ++j) {
                        mma_16816(acc, 0x00010001u, 0x00010001u, 0x00010001u, 0x00010001u, qf[j][0], qf[j][1]);
                        mma_16816(acc, 0x00100010u, 0x00100010u, 0x00100010u, 0x00100010u, qf[j][2], qf[j][3]);
                    }
#pragma unroll
                    for (int i = 0; i < NV; ++i) qsum[g][i] = PARTS ? acc[0] + acc[1] : acc[i];
                }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    f[i] = __shfl_sync(0xffffffffu, ff, (2 * tig + i) * 4);  // from a lane of column 2 tig + i
                    const int rr = row0 + (WIDE ? tig : 2 * tig + i);
                    lim[i] = rr < a.R ? len - (a.T - 1 - token_of(rr)) : 0;
                }
            }
            auto sees = [&](int i) { return BOTH ? __float_as_int(q_row[(i >> 1) * 8 + (i & 1)].y) : lim[BOTH ? 0 : i]; };
            auto row_of = [&](int i) { return row0 + (WIDE ? tig : (i >> 1) * 8 + 2 * tig + (i & 1)); };
            // this lane's logits of its first row; row_of(i) - row_of(0) rows further on the others'
            float* const lg = a.logits + (((size_t)b * c.H + h) * a.R + row_of(0)) * c.cap + tok0;
            const int all_see = len - (a.T - 1);             // slots below this are seen by every row

            float o[TL][H32][2][4], om[BOTH ? 1 : NG][NV], sum_ps[BOTH ? 1 : NG][NV], l[NV], mx[NV];
            int centre = kAttnCentre;
            // The weights enter the second product as p s in fp16.  mx is the largest logit + log2 s (s: a slot's largest scale)
            // that the row has met, moved only when exceeded by kAttnRoom, and p is 2^(logit - mx + 8): a row's largest p s
            // stands between 2^8 and 2^12 and keeps its bits, whatever the scales of slots that it gives no weight or does not
            // see.  (Under one power for a warp's slots, a row lost them with values 1e-4 times the others'.)
            // Two parts carry 22 bits of p s from 2^-3 up, so a group whose scale is 2^-11 of the slot's largest keeps them too
            // (high parts as multiples of 2^-2, whose sums would be exact, kept 2^-24 of the largest only: 1e-4 at a ratio of 1e-3,
            // and 4e-7 against 3e-7 where groups are alike).
            // kRows16 follows p 2^k likewise, 2^k the power of a slot's values: 2^(8 + 6) at most.
            constexpr float E = 8.f;
#pragma unroll
            for (int tl = 0; tl < TL; ++tl)
#pragma unroll
                for (int j = 0; j < H32; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[tl][j][0][e] = o[tl][j][1][e] = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                l[i] = 0.f;
                mx[i] = kNoLogit;
#pragma unroll
                for (int g = 0; g < (BOTH ? 1 : NG); ++g) om[g][i] = sum_ps[g][i] = 0.f;
            }

            const int seg_end = (first_tile + n_tiles) * TILE < len ? (first_tile + n_tiles) * TILE : len;
            for (int n0 = first_tile * TILE + sg * CH; n0 < seg_end; n0 += stride) {
                {
                    uint8_t* kst = enter();
                    // ---- logits: S^T [UN][16 slots][8 columns]; lo[u][v]: slot n0 + 16 u + 8 v + tok0 ----
                    const int na = n0 + tok0;
                    const bool edge = n0 + CH > all_see;     // some row does not see some slot
#pragma unroll 1
                    for (int e = edge; e; e = opaque_zero()) {               // pairs beyond the sequence may be anything: zero them
                        for (int i = lane; i < CH * NG; i += 32)
                            if (n0 + i / NG >= len) reinterpret_cast<uint32_t*>(kst + CODES)[i] = 0u;
                        __syncwarp();
                    }
                    float lo[UN][2][NV];
                    if constexpr (BOTH) {
                        static_assert(!BOTH || (UN == 1 && NG >= 4), "one piece of 16 slots at a time, pairs of a slot in two lanes");
                        const uint8_t *krow = kst + tok0 * CODE_ROW + tig * (D / 8), *kpr = kst + CODES + tok0 * PAIR_ROW;
                        uint32_t w0[D / 32], w1[D / 32], kp0[NG], kp1[NG];
                        ld_words<D / 32>(w0, krow);
                        ld_words<D / 32>(w1, krow + 8 * CODE_ROW);
                        ld_words<NG>(kp0, kpr);
                        ld_words<NG>(kp1, kpr + 8 * PAIR_ROW);
                        // o_g sum q of all groups in one MMA: offsets of groups 2 tig and 2 tig + 1 against the sums' two parts
                        uint32_t o0 = 0u, o1 = 0u;
                        if (2 * tig < NG) {
                            const uint2 p0 = *reinterpret_cast<const uint2*>(kpr + 8 * tig), p1 = *reinterpret_cast<const uint2*>(kpr + 8 * PAIR_ROW + 8 * tig);
                            o0 = __byte_perm(p0.x, p0.y, 0x7632);
                            o1 = __byte_perm(p1.x, p1.y, 0x7632);
                        }
#pragma unroll
                        for (int tl = 0; tl < TL; ++tl) {
                            float off[4];
                            const uint2 sums = q_sums[tl * 32];
                            mma_16816_zero(off, o0, o1, o0, o1, sums.x, sums.y);
#pragma unroll
                            for (int e = 0; e < 4; ++e) lo[0][e >> 1][2 * tl + (e & 1)] = off[e] * (1.f / kCodeScaleLow);
                        }
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            float acc[TL][4];
#pragma unroll
                            for (int j = g * G / 32; j < (g + 1) * G / 32; ++j) {
                                const uint32_t x0 = code_word<G, H32>(w0, j), x1 = code_word<G, H32>(w1, j);
                                const uint32_t y0 = x0 >> 8, y1 = x1 >> 8;
                                const uint32_t e0 = x0 & 0x000f000fu, e1 = x1 & 0x000f000fu, e2 = y0 & 0x000f000fu, e3 = y1 & 0x000f000fu;
                                const uint32_t d0 = x0 & 0x00f000f0u, d1 = x1 & 0x00f000f0u, d2 = y0 & 0x00f000f0u, d3 = y1 & 0x00f000f0u;
#pragma unroll
                                for (int tl = 0; tl < TL; ++tl) {
                                    const uint4 q = q_frag[(tl * H32 + j) * 32];
                                    if (j == g * G / 32) mma_16816_zero(acc[tl], e0, e1, e2, e3, q.x, q.y);
                                    else mma_16816(acc[tl], e0, e1, e2, e3, q.x, q.y);
                                    mma_16816(acc[tl], d0, d1, d2, d3, q.z, q.w);
                                }
                            }
                            const float s0 = pair_f32(kp0[g]).x, s1 = pair_f32(kp1[g]).x;
#pragma unroll
                            for (int i = 0; i < NV; ++i) {
                                lo[0][0][i] = fmaf(s0, acc[i >> 1][i & 1], lo[0][0][i]);
                                lo[0][1][i] = fmaf(s1, acc[i >> 1][2 + (i & 1)], lo[0][1][i]);
                            }
                        }
                    } else {
#pragma unroll
                    for (int u = 0; u < UN; ++u) {
                        const uint8_t* krow = kst + (u * 16 + tok0) * CODE_ROW + tig * (D / 8);
                        uint32_t w0[D / 32], w1[D / 32], kp0[NG], kp1[NG];
                        ld_words<D / 32>(w0, krow);
                        ld_words<D / 32>(w1, krow + 8 * CODE_ROW);
                        const uint8_t* kpr = kst + CODES + (u * 16 + tok0) * PAIR_ROW;
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
                            float2 p0 = pair_f32(kp0[g]), p1 = pair_f32(kp1[g]);
                            if (CENTRED) {
                                p0.y = fmaf(8.f, p0.x, p0.y);
                                p1.y = fmaf(8.f, p1.x, p1.y);
                            }
#pragma unroll
                            for (int i = 0; i < NV; ++i) {
                                if (CENTRED) {               // the sums of high parts are exact: what cancels leaves nothing behind
                                    acc[0] = fmaf(-8.f, qsum[g][0], acc[0]);
                                    acc[2] = fmaf(-8.f, qsum[g][0], acc[2]);
                                }
                                const float a0 = PARTS ? acc[0] + acc[1] : acc[i], a1 = PARTS ? acc[2] + acc[3] : acc[2 + i];
                                const float o0 = p0.y * qsum[g][i], o1 = p1.y * qsum[g][i];
                                lo[u][0][i] = fmaf(p0.x, a0, g ? lo[u][0][i] + o0 : o0);
                                lo[u][1][i] = fmaf(p1.x, a1, g ? lo[u][1][i] + o1 : o1);
                            }
                        }
                    }
                    }
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const float by = BOTH ? q_row[(i >> 1) * 8 + (i & 1)].x : f[BOTH ? 0 : i];
#pragma unroll
                        for (int u = 0; u < UN; ++u)
#pragma unroll
                            for (int v = 0; v < 2; ++v) lo[u][v][i] *= by;
                    }
                    if (a.accumulate) {
                        // what a row does not see may be written too: it lies within the capacity and is never read
#pragma unroll
                        for (int i = 0; i < NV; ++i)
                            if (row_of(i) < a.R) {
                                float* to = lg + (size_t)(row_of(i) - row_of(0)) * c.cap + n0;
#pragma unroll
                                for (int u = 0; u < UN; ++u)
                                    if (UN == 1 || u == 0 || n0 + 16 < len) {
                                        to[16 * u] = lo[u][0][i];
                                        to[16 * u + 8] = lo[u][1][i];
                                    }
                            }
                    }
#pragma unroll 1
                    for (int e = edge; e; e = opaque_zero()) {
#pragma unroll
                        for (int i = 0; i < NV; ++i)
#pragma unroll
                            for (int u = 0; u < UN; ++u)
#pragma unroll
                                for (int v = 0; v < 2; ++v)
                                    if (na + 16 * u + 8 * v >= sees(i)) lo[u][v][i] = -__int_as_float(0x7f800000);
                    }
                    leave(0);
                    uint8_t* vst = enter();
                    // ---- value pairs, running maximum ----
                    uint32_t vp[UN][2][NG];
                    float most[NV], down[2] = {1.f, 1.f};
                    if constexpr (BOTH) {
                        uint32_t* const pairs = reinterpret_cast<uint32_t*>(vst + CODES);
                        auto is_nan = [](uint32_t w) { return (w & 0x7fffu) > 0x7c00u || (w & 0x7fff0000u) > 0x7c000000u; };
#pragma unroll 1
                        for (int e = edge; e; e = opaque_zero()) {
                            // Slots beyond the sequence count for nothing.  A NaN in a slot that some rows do not see goes to the
                            // outputs of those that do here, and not through the MMA, where it would reach all.
                            for (int i0 = 0; i0 < CH * NG; i0 += 32) {
                                const int i = i0 + lane, n = n0 + i / NG;
                                const uint32_t w = i < CH * NG ? pairs[i] : 0u;
                                const bool bad = i < CH * NG && n >= all_see && n < len && is_nan(w);
                                if (i < CH * NG && (n >= len || bad)) pairs[i] = 0u;
                                for (unsigned left = __ballot_sync(0xffffffffu, bad); left; left &= left - 1u) {
                                    const int at = i0 + __ffs(left) - 1;
#pragma unroll
                                    for (int r = 0; r < NV; ++r) {
                                        const bool seen = n0 + at / NG < sees(r);
#pragma unroll
                                        for (int j = 0; j < H32; ++j) {
                                            const float more = seen && j * 32 / G == at % NG ? __int_as_float(0x7fffffff) : 0.f;
#pragma unroll
                                            for (int d = 0; d < 4; ++d) o[r >> 1][j][d >> 1][2 * (d & 1) + (r & 1)] += more;
                                        }
                                    }
                                }
                            }
                            __syncwarp();
                        }
                        // Every slot's pairs to a power of two: the largest s or |o| into [2^6, 2^7), so that 16 |s c + o| stays
                        // below 2^15; p takes the power, and its reference follows p 2^k.  A lane per half a slot.
                        constexpr int WORDS = NG / 2;
                        const int slot = lane >> 1;
                        uint32_t w[WORDS];
                        uint32_t* const at = pairs + slot * NG + (lane & 1) * WORDS;
                        ld_words<WORDS>(w, reinterpret_cast<const uint8_t*>(at));
                        __half2 m = __float2half2_rn(0.f);   // a NaN counts as nothing: of it and a number, the number is the larger one
#pragma unroll
                        for (int i = 0; i < WORDS; ++i) m = __hmax2(m, __habs2(as_half2(w[i])));
                        uint32_t bits = as_word(m) & 0xffffu;
                        bits = bits > as_word(m) >> 16 ? bits : as_word(m) >> 16;
                        const uint32_t other = __shfl_xor_sync(0xffffffffu, bits, 1);
                        bits = bits > other ? bits : other;
                        int e = (int)(bits >> 10);           // its exponent + 15; 31 (an infinity) is not in the format
                        e = e == 31 || e < 6 ? 6 : e;
                        const uint32_t factor = (uint32_t)(36 - e) * 0x04000400u;            // 2^(21 - e) twice
#pragma unroll
                        for (int i = 0; i < WORDS; ++i) at[i] = as_word(__hmul2(as_half2(w[i]), as_half2(factor)));
                        if ((lane & 1) == 0) slot_power[slot] = make_float2((float)(e - 14), pow2(14 - e));
                        __syncwarp();
                        const float2 power[2] = {slot_power[tok0], slot_power[tok0 + 8]};
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            lo[0][0][i] += power[0].x;
                            lo[0][1][i] += power[1].x;
                            most[i] = fmaxf(lo[0][0][i], lo[0][1][i]);
                        }
                        down[0] = power[0].y;
                        down[1] = power[1].y;
                    } else {
#pragma unroll
                    for (int u = 0; u < UN; ++u)
#pragma unroll
                        for (int v = 0; v < 2; ++v) ld_words<NG>(vp[u][v], vst + CODES + (16 * u + 8 * v + tok0) * PAIR_ROW);
#pragma unroll 1
                    for (int e = edge; e; e = opaque_zero()) {
                        // A slot beyond the sequence counts for nothing, whatever it holds; nor does one that a lane's one
                        // column does not see (of two columns, one may: they are told apart below).
#pragma unroll
                        for (int u = 0; u < UN; ++u)
#pragma unroll
                            for (int v = 0; v < 2; ++v)
#pragma unroll
                                for (int g = 0; g < NG; ++g)
                                    if (na + 16 * u + 8 * v >= (WIDE ? lim[0] : len)) vp[u][v][g] = 0u;
                    }
#pragma unroll
                    for (int i = 0; i < NV; ++i) most[i] = -__int_as_float(0x7f800000);
#pragma unroll
                    for (int u = 0; u < UN; ++u)
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            __half2 s = as_half2(0x00010001u);           // 2^-24, the smallest number: for scales that are 0 or NaN
#pragma unroll
                            for (int g = 0; g < NG; ++g) s = __hmax2(s, as_half2(vp[u][v][g]));
                            const float k = log2_fast(__low2float(s));
#pragma unroll
                            for (int i = 0; i < NV; ++i) most[i] = fmaxf(most[i], lo[u][v][i] + k);
                        }
                    }
                    bool change = false;
#pragma unroll
                    for (int i = 0; i < NV; ++i) change |= most[i] > mx[i] + kAttnRoom<MODE>;
                    if (__any_sync(0xffffffffu, change)) {
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            float m = most[i];
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                            if (BOTH) m = ceilf(m);          // a whole number, as k is: their difference is exact
                            m = fmaxf(m, mx[i]);
                            const float corr = exp2_fast(mx[i] - m);
                            mx[i] = m;
                            l[i] *= corr;
#pragma unroll
                            for (int g = 0; g < (BOTH ? 1 : NG); ++g) {
                                om[g][i] *= corr;
                                sum_ps[g][i] *= corr;
                            }
#pragma unroll
                            for (int j = 0; j < H32; ++j)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    o[i >> 1][j][e][i & 1] *= corr;
                                    o[i >> 1][j][e][2 + (i & 1)] *= corr;
                                    if (PARTS) {
                                        o[0][j][e][1] *= corr;
                                        o[0][j][e][3] *= corr;
                                    }
                                }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const float ref = mx[i] - E;
#pragma unroll
                        for (int u = 0; u < UN; ++u)
#pragma unroll
                            for (int v = 0; v < 2; ++v) {
                                lo[u][v][i] = exp2_fast(lo[u][v][i] - ref);          // p from here on
                                l[i] = BOTH ? fmaf(lo[u][v][i], down[v], l[i]) : l[i] + lo[u][v][i];
                            }
                    }
                    // ---- O^T += V^T P^T, per group of scales ----
                    if constexpr (BOTH) {
                        uint32_t bf[TL][2];
#pragma unroll
                        for (int tl = 0; tl < TL; ++tl)
#pragma unroll
                            for (int v = 0; v < 2; ++v) bf[tl][v] = movmatrix_trans(pack_half2(lo[0][v][2 * tl], lo[0][v][2 * tl + 1]));
                        const uint8_t *vrow = vst + tig * CODE_ROW + gid * (D / 16), *vpr = vst + CODES + tig * PAIR_ROW;
                        uint32_t va[H32 / 2], vb[H32 / 2], vc[H32 / 2], vd[H32 / 2];
                        ld_words<H32 / 2>(va, vrow);
                        ld_words<H32 / 2>(vb, vrow + 4 * CODE_ROW);
                        ld_words<H32 / 2>(vc, vrow + 8 * CODE_ROW);
                        ld_words<H32 / 2>(vd, vrow + 12 * CODE_ROW);
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            // the slots of an entry pair: tig and tig + 4, tig + 8 and tig + 12
                            uint32_t pr[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) pr[e] = *reinterpret_cast<const uint32_t*>(vpr + 4 * e * PAIR_ROW + 4 * g);
                            __half2 sc[2], even[2], odd[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                sc[e] = as_half2(__byte_perm(pr[2 * e], pr[2 * e + 1], 0x5410));
                                even[e] = __hfma2(sc[e], __float2half2_rn(8.f), as_half2(__byte_perm(pr[2 * e], pr[2 * e + 1], 0x7632)));
                                odd[e] = __hmul2(even[e], __float2half2_rn(16.f));
                            }
                            auto value = [&](uint32_t x, int e) { return as_word(__hfma2(as_half2(centred<0x000f000fu>(x, above)), sc[e], even[e])); };
                            auto value16 = [&](uint32_t x, int e) { return as_word(__hfma2(as_half2(centred<0x00f000f0u>(x, above)), sc[e], odd[e])); };
#pragma unroll
                            for (int j = g * G / 32; j < (g + 1) * G / 32; ++j) {
                                const uint32_t x = __byte_perm(va[j / 2], vb[j / 2], j & 1 ? 0x7632 : 0x5410);
                                const uint32_t y = __byte_perm(vc[j / 2], vd[j / 2], j & 1 ? 0x7632 : 0x5410);
                                const uint32_t x8 = x >> 8, y8 = y >> 8;
                                {
                                    const uint32_t a0 = value(x, 0), a1 = value(x8, 0), a2 = value(y, 1), a3 = value(y8, 1);
#pragma unroll
                                    for (int tl = 0; tl < TL; ++tl) mma_16816(o[tl][j][0], a0, a1, a2, a3, bf[tl][0], bf[tl][1]);
                                }
                                const uint32_t a0 = value16(x, 0), a1 = value16(x8, 0), a2 = value16(y, 1), a3 = value16(y8, 1);
#pragma unroll
                                for (int tl = 0; tl < TL; ++tl) mma_16816(o[tl][j][1], a0, a1, a2, a3, bf[tl][0], bf[tl][1]);
                            }
                        }
                    } else {
#pragma unroll
                    for (int u = 0; u < UN; ++u) {
                        const uint8_t* vrow = vst + (u * 16 + tig) * CODE_ROW + gid * (D / 16);
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
                                uint32_t pair = vp[u][v][RELOAD ? 0 : g];
                                if (RELOAD) {
                                    pair = *reinterpret_cast<const uint32_t*>(vst + CODES + (16 * u + 8 * v + tok0) * PAIR_ROW + 4 * g);
                                    if (edge && na + 16 * u + 8 * v >= (WIDE ? lim[0] : len)) pair = 0u;
                                }
                                const float2 so = pair_f32(pair);
                                float ps[NV];
                                float om_was[NV];
#pragma unroll
                                for (int i = 0; i < NV; ++i) {
                                    om_was[i] = om[g][i];
                                    ps[i] = lo[u][v][i] * so.x;
                                    om[g][i] = fmaf(lo[u][v][i], PARTS ? fmaf(8.f, so.x, so.y) : so.y, om[g][i]);
                                }
                                if (!WIDE && edge) {         // a slot that a row does not see adds nothing, whatever it holds
#pragma unroll
                                    for (int i = 0; i < NV; ++i)
                                        if (na + 16 * u + 8 * v >= lim[i]) {
                                            ps[i] = 0.f;
                                            om[g][i] = om_was[i];
                                        }
                                }
#pragma unroll
                                for (int i = 0; i < NV; ++i)
                                    if (!PARTS) sum_ps[g][i] += ps[i];
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
                                if (PARTS) {
                                    mma_16816(o[0][j][0], centred<0x000f000fu>(x, above), centred<0x000f000fu>(x8, above),
                                              centred<0x000f000fu>(y, above), centred<0x000f000fu>(y8, above), bf[0], bf[1]);
                                    mma_16816(o[0][j][1], centred<0x00f000f0u>(x, above), centred<0x00f000f0u>(x8, above),
                                              centred<0x00f000f0u>(y, above), centred<0x00f000f0u>(y8, above), bf[0], bf[1]);
                                } else {
                                    mma_16816(o[0][j][0], x & 0x000f000fu, x8 & 0x000f000fu, y & 0x000f000fu, y8 & 0x000f000fu, bf[0], bf[1]);
                                    mma_16816(o[0][j][1], x & 0x00f000f0u, x8 & 0x00f000f0u, y & 0x00f000f0u, y8 & 0x00f000f0u, bf[0], bf[1]);
                                }
                            }
                        }
                    }
                    }
                }
                leave(1);
                if (!PARTS && !BOTH && --centre == 0) {
                    centre = kAttnCentre;
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        // what is taken out and put back is one fp16 number per lane, so the two are the same; the rest waits
                        float take[NV];
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            take[i] = __half2float(__float2half_rn(fminf(sum_ps[g][i], 60000.f)));
                            sum_ps[g][i] -= take[i];
                            om[g][i] = fmaf(8.f, take[i], om[g][i]);
                        }
                        const uint32_t b0 = movmatrix_trans(pack_half2(take[0], WIDE ? 0.f : take[NV - 1]));
#pragma unroll
                        for (int j = g * G / 32; j < (g + 1) * G / 32; ++j) {
                            mma_16816(o[0][j][0], 0x80088008u, 0x80088008u, 0x80088008u, 0x80088008u, b0, 0u);
                            mma_16816(o[0][j][1], 0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u, b0, 0u);
                        }
                    }
                }
            }

            // ---- join the warps of a row tile, JOIN rows of it at a time ----
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
#pragma unroll
                    for (int g = 0; g < (BOTH ? 1 : NG); ++g) om[g][i] += __shfl_xor_sync(0xffffffffu, om[g][i], d);
                }
            }
            const Cursor was = k;
            const bool whole = n_tiles == was.nt;
            const int piece = blockIdx.x * 2 + (first_tile == 0 ? 1 : 0);
#pragma unroll
            for (int tl = 0; tl < TL; ++tl) {
                __syncthreads();                             // the buffer's last use is over
#pragma unroll
                for (int i = 0; i < NV / TL; ++i) {
                    const int ii = tl * 2 + i, r = WIDE ? tig : 2 * tig + i;
                    if (gid == 0) mlbuf[warp * JOIN + r] = make_float2(mx[ii] - E, l[ii]);
#pragma unroll
                    for (int j = 0; j < H32; ++j) {
                        const float add = BOTH ? 0.f : om[BOTH ? 0 : j * 32 / G][ii];
                        float4 v;
                        if (PARTS) {
                            v.x = o[tl][j][0][0] + o[tl][j][0][1];
                            v.y = o[tl][j][1][0] + o[tl][j][1][1];
                            v.z = o[tl][j][0][2] + o[tl][j][0][3];
                            v.w = o[tl][j][1][2] + o[tl][j][1][3];
                        } else {
                            v.x = o[tl][j][0][i];
                            v.y = o[tl][j][1][i];
                            v.z = o[tl][j][0][2 + i];
                            v.w = o[tl][j][1][2 + i];
                        }
                        // kRows16: values entered with 2^(7 - k)
                        constexpr float even = BOTH ? 1.f / 128.f : (PARTS ? 1.f : kCodeScaleLow), odd = BOTH || PARTS ? even / 16.f : kCodeScaleHigh;
                        v.x = fmaf(v.x, even, add);
                        v.y = fmaf(v.y, odd, add);
                        v.z = fmaf(v.z, even, add);
                        v.w = fmaf(v.w, odd, add);
                        *reinterpret_cast<float4*>(obuf + ((size_t)warp * JOIN + r) * D + j * 32 + gid * 4) = v;
                    }
                }
                __syncthreads();
                if (tl == 0 && t + n_tiles < n_total) {      // the next unit's query rows are on their way during the join
                    k = advance(k, n_tiles);
                    load_q(k);
                }
                // `lanes` neighbouring lanes take the nsg parts of one quad of outputs in turn, and add them up by shuffles: as
                // many as leave no lane without a quad (15 rows of 128: 1100 instructions a warp with 8, 250 with 1)
                const int rows_here = a.R - rb * a.RU < a.RU ? a.R - rb * a.RU : a.RU;
                const int items = (BOTH ? a.RT * JOIN : rows_here) * (D / 4);
                int lanes = nsg;
                while (lanes > 1 && items * lanes > kAttnThreads) lanes >>= 1;
                const int part = tid & (lanes - 1), per_round = kAttnThreads / lanes;
                for (int i0 = 0; i0 < items; i0 += per_round) {
                    const int item = i0 + tid / lanes, at = item < items ? item / (D / 4) : 0, d4 = item % (D / 4);
                    const int ru = BOTH ? at / JOIN * RPT + tl * JOIN + at % JOIN : at;
                    const int from = (part * a.RT + at / JOIN) * JOIN + at % JOIN, step = lanes * a.RT * JOIN;       // row of the part's warp
                    float top = kNoLogit * 2.f;
                    for (int q = part, r = from; q < nsg; q += lanes, r += step) top = fmaxf(top, mlbuf[r].x);
                    for (int d = 1; d < lanes; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    float sum = 0.f;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int q = part, r = from; q < nsg; q += lanes, r += step) {
                        const float2 ml = mlbuf[r];
                        const float4 x = *reinterpret_cast<const float4*>(obuf + (size_t)r * D + d4 * 4);
                        const float e = exp2_fast(ml.x - top);
                        sum = fmaf(ml.y, e, sum);
                        v.x = fmaf(x.x, e, v.x);
                        v.y = fmaf(x.y, e, v.y);
                        v.z = fmaf(x.z, e, v.z);
                        v.w = fmaf(x.w, e, v.w);
                    }
                    for (int d = 1; d < lanes; d <<= 1) {
                        sum += __shfl_xor_sync(0xffffffffu, sum, d);
                        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
                        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
                        v.z += __shfl_xor_sync(0xffffffffu, v.z, d);
                        v.w += __shfl_xor_sync(0xffffffffu, v.w, d);
                    }
                    if (part != 0 || item >= items || ru >= rows_here) continue;
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
            }
            t += n_tiles;
        }
    }
}

// ------------------------------------------------------------------------------ finish --
// Blocks x < R of a (sequence, head): query row x, joined from the pieces of its unit where that was cut
// (zeros where the sequence is empty).  Blocks beyond: finish_slots slots each, whose weights get the
// sum over rows of 2^(logit - maximum) / sum.  A thread has U quads of slots and BATCH rows in flight: 4 and 1 where
// there is one row per key head, else 1 and 8.  Bound by latency (4 to 5 us beside the attention kernel at 8 x 32 heads x
// 4001), and by the bytes of the logits, which come from L2, where there are many rows.
constexpr int kFinishThreads = 256;
constexpr int kFinishSlots = 4 * kFinishThreads;             // per round of a block

template <typename T, int U, int BATCH>
__global__ void __launch_bounds__(kFinishThreads, 3) kv4_finish_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    const Kv4& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_number(), h = blockIdx.y, b = blockIdx.z, D = c.D;
    const size_t unit0 = ((size_t)b * c.H + h) * a.RB;
    wait_for_stream();
    let_next_start();
    const int len = kv4_length(c, b);

    if ((int)blockIdx.x < a.R) {
        const int r = blockIdx.x, rb = r / a.RU, ru = r % a.RU;
        const int rt_ = a.T == 1 ? 0 : r / a.share;
        T* dst = (T*)a.out + ((long long)b * a.T + rt_) * a.ld_out + (long long)(h * a.share + r - rt_ * a.share) * D;
        if (len == 0) {
            for (int d = tid; d < D; d += kFinishThreads) dst[d] = from_f32<T>(0.f);
            return;
        }
        const int2 range = a.pieces[unit0 + rb];
        const int i0 = range.x, i1 = range.y;
        if (i0 == i1) return;
        const int n = i1 - i0 + 1;
        auto piece = [&](int i) { return ((size_t)(i0 + i) * 2 + (i == 0 ? 1 : 0)) * a.RU + ru; };
        float top = kNoLogit * 2.f, sum = 0.f;               // every warp for itself
        for (int i = lane; i < n; i += 32) top = fmaxf(top, a.part_ml[piece(i)].x);
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        for (int i = lane; i < n; i += 32) {
            const float2 ml = a.part_ml[piece(i)];
            sum = fmaf(ml.y, exp2_fast(ml.x - top), sum);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        // D / 4 threads cover the row, 256 / (D / 4) of such groups take the pieces in turn
        const int quads = D / 4, groups = kFinishThreads / quads, d4 = tid % quads, g = tid / quads;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = g; i < n; i += groups) {
            const float4 x = *reinterpret_cast<const float4*>(a.part_o + piece(i) * D + d4 * 4);
            const float e = exp2_fast(a.part_ml[piece(i)].x - top);
            v.x = fmaf(x.x, e, v.x);
            v.y = fmaf(x.y, e, v.y);
            v.z = fmaf(x.z, e, v.z);
            v.w = fmaf(x.w, e, v.w);
        }
        float4* buf = reinterpret_cast<float4*>(smem);
        buf[tid] = v;
        __syncthreads();
        if (g == 0) {
            for (int j = 1; j < groups && j < n; ++j) {
                const float4 x = buf[j * quads + d4];
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            store4(dst + d4 * 4, v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        }
        return;
    }

    // weights: four slots a thread (the capacity is a multiple of 16, so they lie within a row of logits); the first rows'
    // logits are on their way while the rows' maxima and sums are put together
    const int first = ((int)blockIdx.x - a.R) * a.finish_slots, end = first + a.finish_slots < len ? first + a.finish_slots : len;
    if (first >= end) return;
    const float* lg = a.logits + ((size_t)b * c.H + h) * a.R * c.cap;
    float* weight = c.weight + ((size_t)b * c.H + h) * c.cap;
    float4 w[U], x[U][BATCH];
    auto load_w = [&](int n0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (n0 + u * kFinishSlots < end) w[u] = *reinterpret_cast<const float4*>(weight + n0 + u * kFinishSlots);
    };
    auto load_x = [&](int n0, int r0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < BATCH; ++k)
                if (n0 + u * kFinishSlots < end && r0 + k < a.R)
                    x[u][k] = *reinterpret_cast<const float4*>(lg + (size_t)(r0 + k) * c.cap + n0 + u * kFinishSlots);
    };
    load_w(first + tid * 4);
    load_x(first + tid * 4, 0);
    // maximum and 1 / sum of every row, and how many slots it sees; one warp per row
    float2* rows = reinterpret_cast<float2*>(smem);                      // [R]
    int* sees = reinterpret_cast<int*>(rows + a.R);                      // [R]
    int rb = -1, i0 = 0, i1 = 0;
    for (int r = warp; r < a.R; r += kFinishThreads / 32) {
        const int of = a.RB == 1 ? 0 : r / a.RU, ru = r - of * a.RU;
        if (of != rb) {
            rb = of;
            const int2 range = a.pieces[unit0 + rb];
            i0 = range.x;
            i1 = range.y;
        }
        float top, sum;
        if (i0 == i1) {
            const float2 ml = a.stats[(unit0 + rb) * a.RU + ru];
            top = ml.x;
            sum = ml.y;
        } else {
            float2 ml = make_float2(kNoLogit * 2.f, 0.f);                // up to 32 pieces are loaded once
            if (i0 + lane <= i1) ml = a.part_ml[((size_t)(i0 + lane) * 2 + (lane == 0)) * a.RU + ru];
            top = ml.x;
            for (int i = i0 + lane + 32; i <= i1; i += 32) top = fmaxf(top, a.part_ml[(size_t)i * 2 * a.RU + ru].x);
#pragma unroll
            for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            sum = ml.y * exp2_fast(ml.x - top);
            for (int i = i0 + lane + 32; i <= i1; i += 32) {
                const float2 more = a.part_ml[(size_t)i * 2 * a.RU + ru];
                sum = fmaf(more.y, exp2_fast(more.x - top), sum);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        }
        if (lane == 0) {
            rows[r] = make_float2(top, sum == 0.f ? 0.f : 1.f / sum);
            sees[r] = len - (a.T - 1 - (a.T == 1 ? 0 : r / a.share));
        }
    }
    __syncthreads();
    for (int n0 = first + tid * 4; n0 < end; n0 += U * kFinishSlots) {
        if (n0 >= first + U * kFinishSlots) {
            load_w(n0);
            load_x(n0, 0);
        }
        // several rows are added up by themselves: one rounding of the weight, however large it is already
        float4 add[U];
#pragma unroll
        for (int u = 0; u < U; ++u) add[u] = BATCH == 1 ? w[u] : make_float4(0.f, 0.f, 0.f, 0.f);
        for (int r0 = 0; r0 < a.R; r0 += BATCH) {
            if (r0 > 0) load_x(n0, r0);
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                if (r0 + k >= a.R) break;
                const float2 ml = rows[r0 + k];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int see = sees[r0 + k] - (n0 + u * kFinishSlots);          // slots of the four that the row sees
                    if (see > 0) add[u].x = fmaf(exp2_fast(x[u][k].x - ml.x), ml.y, add[u].x);
                    if (see > 1) add[u].y = fmaf(exp2_fast(x[u][k].y - ml.x), ml.y, add[u].y);
                    if (see > 2) add[u].z = fmaf(exp2_fast(x[u][k].z - ml.x), ml.y, add[u].z);
                    if (see > 3) add[u].w = fmaf(exp2_fast(x[u][k].w - ml.x), ml.y, add[u].w);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (n0 + u * kFinishSlots < end)
                *reinterpret_cast<float4*>(weight + n0 + u * kFinishSlots) =
                    BATCH == 1 ? add[u] : make_float4(w[u].x + add[u].x, w[u].y + add[u].y, w[u].z + add[u].z, w[u].w + add[u].w);
    }
}

// -------------------------------------------------------------------------------- host --
static inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Shared memory of the main kernel: rings, the join of the warps, the laid-out query rows of `query_tiles` row tiles (16-row form
// only: 0 elsewhere) and the lists of sequences.
static inline size_t attn_smem(const Kv4& c, int stages, int tile, int join_rows, int query_tiles)
{
    const size_t ring = (size_t)stages * (tile / kAttnWarps) * (c.D / 2 + c.D / c.G * 4);
    const size_t query = 2 * (c.D / 32) * 512 + 2 * 256 + 16 * 8;
    return kAttnWarps * (ring + join_rows * (c.D * sizeof(float) + sizeof(float2))) +
           (query_tiles ? query_tiles * query + kAttnWarps * 16 * sizeof(float2) : 0) + (3 * c.B + 1) * sizeof(int);
}

// Row tiles per unit, rows per unit and units per key head for R query rows: the split with the least work.  A tile of
// rows costs the same wherever it is (its warps copy the codes for themselves, from L2), so padding decides over long caches; a unit
// costs some tiles more, and the CTAs end apart by a tile of all the unit's rows.  (With as many rows per unit as eight
// warps take: 16 sequences x 35 fp16 rows x 20000 slots 296 us, 173 now; 4 x 8 heads x 56 bf16 rows x 2000 64, 51 now.)
static void attn_rows(const Kv4& c, int R, int rpt, int* RT, int* RU, int* RB)
{
    const int tiles = (R + rpt - 1) / rpt, slots = (c.cap + 255) / 256;
    long long best = 0;
    *RT = 0;
    for (int rt = rpt < 16 ? 8 : 4; rt; rt >>= 1) {          // of 16 rows: two warps per row tile at least
        // where the rows of four tiles do not fit beside the lists of many sequences (head_dim 256 in groups of 32 from batch 512 on)
        if (rpt == 16 && rt > 1 && attn_smem(c, kAttnStages16, kAttnTile16, 8, rt) > kAttnSmemRoom) continue;
        const long long units = (tiles + rt - 1) / rt;
        const long long cost = (long long)c.B * c.H * units * ((long long)rt * slots + 2 * kAttnUnitCost) + (long long)kAttnMaxCtas * rt;
        if (*RT == 0 || cost < best) {
            best = cost;
            *RT = rt;
        }
    }
    *RU = *RT * rpt;
    *RB = (R + *RU - 1) / *RU;
}

struct AttnLayout {
    size_t ml, o, pieces, stats, logits, total;
};
static AttnLayout attn_layout(const Kv4& c, int R, int rpt)
{
    int RT, RU, RB;
    attn_rows(c, R, rpt, &RT, &RU, &RB);
    AttnLayout w;
    w.ml = 0;
    w.o = w.ml + up256((size_t)kAttnMaxCtas * 2 * RU * sizeof(float2));
    w.pieces = w.o + up256((size_t)kAttnMaxCtas * 2 * RU * c.D * sizeof(float));
    w.stats = w.pieces + up256((size_t)c.B * c.H * RB * sizeof(int2));
    w.logits = w.stats + up256((size_t)c.B * c.H * RB * RU * sizeof(float2));
    w.total = w.logits + (c.weight ? up256((size_t)c.B * c.H * R * c.cap * sizeof(float)) : 0);
    return w;
}

template <typename T, int D, int G, int MODE>
static coreinfer_status launch_mode(AttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int TILE = kAttnTile<D, G, MODE>;
    static_assert(kAttnQueryBytes<D> == 2 * (D / 32) * 512 + 2 * 256 + 16 * 8 && kAttnJoinRows<kRows16> == 8, "attn_smem and attn_rows");
    const size_t smem = attn_smem(a.c, kAttnStages<D, G, MODE>, TILE, kAttnJoinRows<MODE>, MODE == kRows16 ? a.RT : 0);
    // two CTAs per SM where registers (head_dim up to 128) and shared memory (batch up to some hundreds) allow it
    const int per_sm = D <= 128 && 2 * (smem + 1024 + 64) <= (size_t)di.smem_optin + 1024 ? 2 : 1;
    if (smem > smem_room(di)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "not enough shared memory");
    const long long tiles = (long long)a.c.B * a.c.H * a.RB * ((a.c.cap + TILE - 1) / TILE + kAttnUnitCost);
    if ((unsigned long long)a.c.B * a.c.H * a.c.cap > 0xffffffffull)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "the cache has more than 2^32 slots");
    if (tiles > (1LL << 30)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "the cache has %lld tiles of %d slots: too many for one call", tiles, TILE);
    long long ctas = (long long)di.sm_count * per_sm;
    if (ctas > kAttnMaxCtas) ctas = kAttnMaxCtas;
    if (ctas > tiles) ctas = tiles;
    a.n_ctas = (int)ctas;
    const coreinfer_status s = allow_smem<kv4_attention_kernel<T, D, G, MODE>>(di);
    if (s != COREINFER_OK) return s;
    CI_CUDA(launch_overlapped(kv4_attention_kernel<T, D, G, MODE>, dim3(a.n_ctas), dim3(kAttnThreads), smem, st, a));
    const size_t join = kFinishThreads * sizeof(float4), rows = (size_t)a.R * (sizeof(float2) + sizeof(int));
    // up to four rounds a block while that leaves about two blocks per SM and slot of it
    a.finish_slots = kFinishSlots;
    while (a.finish_slots < 4 * kFinishSlots &&
           (long long)a.c.B * a.c.H * ((a.c.cap + 2 * a.finish_slots - 1) / (2 * a.finish_slots)) >= 6LL * di.sm_count) a.finish_slots *= 2;
    const dim3 grid(a.R + (a.accumulate ? (a.c.cap + a.finish_slots - 1) / a.finish_slots : 0), a.c.H, a.c.B);
    if (a.R == 1) CI_CUDA(launch_overlapped(kv4_finish_kernel<T, 4, 1>, grid, dim3(kFinishThreads), join > rows ? join : rows, st, a));
    else CI_CUDA(launch_overlapped(kv4_finish_kernel<T, 1, 8>, grid, dim3(kFinishThreads), join > rows ? join : rows, st, a));
    return COREINFER_OK;
}

// Rows per warp for R query rows and `groups` groups per head: fp32 and fp16 always carry two parts; bf16 takes the
// form with four rows where that is enough, and above eight rows the one with sixteen where there are four groups or more
// (4 x 8 heads x up to 4096 slots, 9 / 15 / 24 / 64 rows: head_dim 128 in groups of 32 21.4 / 24.9 / 37.0 / 68.8 us against 22.8 /
// 25.8 / 34.8 / 76.3 with eight rows a warp, so it loses where it pads half a tile; head_dim 256 in groups of 32 31.4 / 35.3 / 51.2 /
// 91.8 against 35.0 / 38.9 / 53.2 / 117; head_dim 128 in groups of 64, where p s is formed for two groups only, 15 / 24 / 64 rows
// of 4096 slots each 23.6 / 32.8 / 57.7 against 21.8 / 30.6 / 55.5).
static inline int attn_rpt(coreinfer_dtype dtype, long long R, int groups)
{
    return dtype != COREINFER_BF16 || R <= 4 ? 4 : (R <= 8 || groups < 4 ? 8 : 16);
}

template <typename T, int D, int G>
static coreinfer_status launch_attention(AttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        if constexpr (D / G >= 4)
            if (a.R > 8) return launch_mode<T, D, G, kRows16>(a, di, st);
        return a.R <= 4 ? launch_mode<T, D, G, kRows4>(a, di, st) : launch_mode<T, D, G, kRows8>(a, di, st);
    } else
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

// The finishing kernel holds 12 bytes per query row in shared memory that needs no opt-in.
static_assert(COREINFER_KV4_MAX_ROWS * (sizeof(float2) + sizeof(int)) <= 48 * 1024, "rows of the finishing kernel");

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

size_t coreinfer_kv4_attention_workspace_bytes(const coreinfer_kv4_cache* cache, int32_t q_heads, int32_t T)
{
    Kv4 c;
    if (kv4_take(cache, "the", &c) != COREINFER_OK) return 0;
    if (q_heads < 1 || T < 1 || q_heads % c.H != 0 || T > COREINFER_KV4_MAX_QUERIES) return 0;
    if ((long long)(q_heads / c.H) * T > COREINFER_KV4_MAX_ROWS) return 0;
    // Fewer rows may take more of them per unit, and the parts of cut units then more bytes: the largest over all types and up to
    // T tokens, so that one workspace serves every shorter call.
    size_t most = 0;
    for (int t = 1; t <= T; ++t)
        for (int rpt = 4; rpt <= 16; rpt *= 2) {
            const size_t n = attn_layout(c, q_heads / c.H * t, rpt).total;
            if (n > most) most = n;
        }
    return most;
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
    if (R > COREINFER_KV4_MAX_ROWS) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%lld query rows per key head: at most %d", R, COREINFER_KV4_MAX_ROWS);
    if (!q || !out || !aligned16(q) || !aligned16(out)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "q / out NULL or not 16-byte aligned");
    const int64_t row = (int64_t)q_heads * a.c.D, e = (int64_t)dtype_size(dtype);
    if (ld_q < row || ld_out < row || (ld_q * e) % 16 != 0 || (ld_out * e) % 16 != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "ld_q and ld_out must cover q_heads * head_dim elements and be multiples of 16 bytes");
    if (accumulate && !a.c.weight) CI_FAIL(COREINFER_ERR_INVALID_ARG, "accumulate needs a cache with weight and position");
    if (!(scale == scale) || scale - scale != 0.f) CI_FAIL(COREINFER_ERR_INVALID_ARG, "scale is not a finite number");
    if (!workspace || !aligned16(workspace)) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace is NULL or misaligned");
    const int rpt = attn_rpt(dtype, R, a.c.D / a.c.G);
    const AttnLayout w = attn_layout(a.c, (int)R, rpt);      // what this call needs, at most what the query says
    if (workspace_bytes < w.total) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, w.total);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    uint8_t* ws = (uint8_t*)workspace;
    a.q = q;
    a.out = out;
    a.ld_q = ld_q;
    a.ld_out = ld_out;
    a.T = T;
    a.share = q_heads / a.c.H;
    a.R = (int)R;
    attn_rows(a.c, a.R, rpt, &a.RT, &a.RU, &a.RB);
    a.scale = scale;
    a.accumulate = accumulate ? 1 : 0;
    a.part_ml = (float2*)(ws + w.ml);
    a.part_o = (float*)(ws + w.o);
    a.pieces = (int2*)(ws + w.pieces);
    a.stats = (float2*)(ws + w.stats);
    a.logits = (float*)(ws + w.logits);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == COREINFER_F32) return pick_attention<float>(a, di, st);
    if (dtype == COREINFER_BF16) return pick_attention<__nv_bfloat16>(a, di, st);
    return pick_attention<__half>(a, di, st);
}

}  // extern "C"
