// Appending to and evicting from the 4-bit key/value cache.
#include "kv4.cuh"

namespace coreinfer {

// -------------------------------------------------------------------------------- append --
// A row is one token's keys or values of one head.  A lane holds eight consecutive values of a row (D / 8 lanes
// per row); the lanes of a group agree on its range by shuffles; neighbouring blocks of 32 values
// exchange a unit so that codes are stored in words.  A CTA walks rows of one sequence so that the sequence's state is
// read, and its ticket taken, a few hundred times at most; a lane moves on by fixed strides and has the next row under way
// while it works on one.  Bound by instructions, about 280 per warp and row of eight values a lane (issue slots 66 % busy): 1000
// tokens x 32 heads x 128 bf16, stored values out, with the launch that clears the state before it 16.7 us from a graph over
// three sets of inputs, 2250 GB/s, and 18.2 on a stream.
constexpr int kAppendThreads = 256;

struct AppendArgs {
    Kv4 c;
    const void* src[2];
    void* stored[2];
    int tokens;
    int rows;               // tokens * H * 2
    long long ld;
};

template <typename T, int D, int G>
__global__ void __launch_bounds__(kAppendThreads) kv4_append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr int LANES = D / 8, ROWS = kAppendThreads / LANES, H32 = D / 32, GL = G / 8;
    const Kv4& c = a.c;
    const int b = blockIdx.y;
    const int l = threadIdx.x % LANES;
    wait_for_stream();
    let_next_start();
    const int4 state = *reinterpret_cast<const int4*>(c.state + b * 4);
    const int n0 = state.x < 0 ? 0 : (state.x > c.cap ? c.cap : state.x), seen = state.y;
    const bool fits = a.tokens <= c.cap - n0;
    // row r holds keys (even r) or values (odd) of head (r / 2) % H of token r / 2 / H; a step is a whole number of tokens,
    // so a lane keeps its head and moves on by fixed strides
    const int row0 = blockIdx.x * ROWS + threadIdx.x / LANES, dt = (int)(gridDim.x * ROWS) / (2 * c.H);
    const int which = row0 & 1, t0 = (row0 >> 1) / c.H, h = (row0 >> 1) - t0 * c.H;
    const bool first = t0 < a.tokens;
    const T* src = (const T*)a.src[which] + ((long long)b * a.tokens + (first ? t0 : 0)) * a.ld + (long long)h * D + l * 8;
    const long long src_step = dt * a.ld;
    size_t slot = ((size_t)b * c.H + h) * c.cap + n0 + t0;
    T* out = (T*)a.stored[which];
    if (out) out += (((long long)b * a.tokens + t0) * c.H + h) * D + l * 8;
    const long long out_step = (long long)dt * c.H * D;
    auto load = [&](const T* p, T (&v)[8]) {
        *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(p);
        if (sizeof(T) == 4) reinterpret_cast<uint4*>(v)[1] = reinterpret_cast<const uint4*>(p)[1];
    };
    T v[8];
    load(src, v);
    int t = t0;
    for (int base = blockIdx.x * ROWS; base < a.rows; base += gridDim.x * ROWS) {             // the same count for a whole CTA
        const bool in = t < a.tokens;
        float x[8], lo, hi;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = to_f32<T>(v[e]);
            lo = e ? min_nan(lo, x[e]) : x[e];
            hi = e ? max_nan(hi, x[e]) : x[e];
        }
        if (t + dt < a.tokens) src += src_step;
        T next[8];
        load(src, next);                                     // on its way while this row is worked on
        group_range(lo, hi, GL);
        const QuantPair p = quant_pair(lo, hi);
        const float s = __half2float(p.s), o = __half2float(p.o);
        unsigned unit[2];
        float q[8];
        quant_codes<8>(x, s, o, unit, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = from_f32<T>(fmaf(s, q[e], o));
        // this lane holds units i = 2 (l % 4), i + 1 of block h32 = l / 4; the lane of block h32 ^ 1 has its neighbours
        const int h32 = l >> 2, odd = h32 & 1;
        const unsigned got = __shfl_xor_sync(0xffffffffu, odd ? unit[0] : unit[1], 4);
        const unsigned word = odd ? got | unit[1] << 16 : unit[0] | got << 16;
        if (in && fits) {
            uint8_t* codes = c.codes[which] + slot * (D / 2);
            *reinterpret_cast<unsigned*>(codes + 2 * ((2 * (l & 3) + odd) * H32 + (h32 & ~1))) = word;
            if (l % GL == 0) c.pairs[which][slot * (D / G) + l / GL] = __halves2half2(p.s, p.o);
            if (!which && l == 0 && c.weight) {
                c.weight[slot] = 0.f;
                c.position[slot] = seen + t;
            }
        }
        if (in && out) {
            *reinterpret_cast<uint4*>(out) = *reinterpret_cast<uint4*>(v);
            if (sizeof(T) == 4) reinterpret_cast<uint4*>(out)[1] = reinterpret_cast<uint4*>(v)[1];
            out += out_step;
        }
        t += dt;
        slot += dt;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = next[e];
    }
    if (kv4_last_of_sequence(c, b, gridDim.x)) {
        if (fits) {
            c.state[b * 4 + kStateLength] = n0 + a.tokens;
            c.state[b * 4 + kStateSeen] = seen + a.tokens;
        } else {
            c.state[b * 4 + kStateRefused] = state.z + a.tokens;
        }
    }
}

template <typename T, int D, int G>
static cudaError_t launch_append(const AppendArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int ROWS = kAppendThreads / (D / 8);
    // CTAs per sequence: a multiple that makes a step a whole number of tokens, about six per SM in all where there is work
    int unit = 2 * a.c.H;
    while (unit > 1 && unit % 2 == 0 && (2 * a.c.H / unit) * 2 <= ROWS) unit /= 2;           // 2 H / gcd(2 H, ROWS), ROWS a power of two
    const long long want = (a.rows + (long long)ROWS * unit - 1) / ((long long)ROWS * unit), most = (di.sm_count * 6 + a.c.B * unit - 1) / (a.c.B * unit);
    return launch_overlapped(kv4_append_kernel<T, D, G>, dim3((unsigned)(want < most ? want : most) * unit, a.c.B), dim3(kAppendThreads), 0, st, a);
}

template <typename T>
static coreinfer_status pick_append(const AppendArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    const int D = a.c.D, G = a.c.G;
    cudaError_t r;
    if (D == 64) r = G == 32 ? launch_append<T, 64, 32>(a, di, st) : launch_append<T, 64, 64>(a, di, st);
    else if (D == 128)
        r = G == 32 ? launch_append<T, 128, 32>(a, di, st) : (G == 64 ? launch_append<T, 128, 64>(a, di, st) : launch_append<T, 128, 128>(a, di, st));
    else
        r = G == 32 ? launch_append<T, 256, 32>(a, di, st) : (G == 64 ? launch_append<T, 256, 64>(a, di, st) : launch_append<T, 256, 128>(a, di, st));
    CI_CUDA(r);
    return COREINFER_OK;
}

// --------------------------------------------------------------------------------- evict --
// kv4_evict_few_kernel, in place with at most 16 slots above the budget (the step of a decode loop at a full budget): one
// CTA per sequence and head takes the smallest key out, once per slot that leaves, and moves what has to move.
// kv4_select_held_kernel, otherwise: one CTA, or a cluster of up to 8 where heads are few and long, per sequence and head.
// Keys (the order of eviction as unsigned numbers) stay in registers, the key of the last slot that stays comes from
// radix selection (11 + 11 + 10 bits, most significant first, stopping as soon as a whole bin stays), then the lists of slots
// that move, by scans over threads and CTAs.
// kv4_select_kernel, more than 16384 slots per CTA: the same with keys in shared memory, or read again for each pass, and
// ballots; a warp owns a contiguous range of slots, so that list order is slot order.
// kv4_move_kernel copies the listed slots, many CTAs per head.
// All are bound by latency at the sizes of a decode step (append and few together 10.2 us for 8 sequences x 32 heads x 2049
// slots from a graph, 10.9 on a stream, of which some 6 are two launches and the reads of the state), the moves by bytes after a
// prompt: 4 x 8 heads x up to 16384 slots down to 2048 in another cache 18.4 us over three sets of inputs (16.9 over two, part of
// which stays in L2), about half of it the selection's barriers and three passes.
constexpr int kEvictBins = 2048;
constexpr int kEvictFew = 16;
constexpr int kEvictKeysMost = 48 * 1024;   // keys a CTA holds in shared memory; more slots are read again for each pass
constexpr int kEvictMaxCluster = 8;
constexpr int kMoveSlots = 64;              // slots per CTA of the moving kernel
constexpr int kMoveThreads = 256;
constexpr int kMoveHere = 64;               // so few slots are moved by the CTA that selected them (room for 45 above the budget: 16.4 us with a
                                            // launch more, 15.2 without; for 256: 13.9 and 20.8)

__device__ __forceinline__ unsigned evict_key(float w, int pos, int seen, int recent, int first)
{
    if (pos >= seen - recent || pos < first) return 0xffffffffu;    // stays for certain: above every number
    if (w != w) return 0u;                                          // NaN: below every number
    const unsigned u = __float_as_uint(w + 0.f);                    // -0 counts as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Copies `count` listed slots; a thread takes one piece of a slot at a time: 16 bytes of codes, or one
// pair, or the weight, or the position.  Sources and destinations do not overlap, so four pieces are read before
// the first is written.
__device__ __forceinline__ void move_slots(const Kv4& a, size_t abase, const Kv4& z, size_t zbase, const int32_t* from, const int32_t* to,
                                           int count, int tid, int threads)
{
    constexpr int U = 4;
    const int chunks = a.D / 32, groups = a.D / a.G, items = 2 * chunks + 2 * groups + 2, all = count * items;
    for (int i0 = tid; i0 < all; i0 += U * threads) {
        uint4 v[U];
        void* dst[U];
        bool wide[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * threads;
            dst[u] = nullptr;
            if (i >= all) continue;
            const int m = i / items;
            int k = i - m * items;
            const size_t s = abase + from[m], d = zbase + to[m];
            const void* src;
            wide[u] = k < 2 * chunks;
            if (wide[u]) {
                const int w = k >= chunks;
                k -= w * chunks;
                src = reinterpret_cast<const uint4*>(a.codes[w] + s * (a.D / 2)) + k;
                dst[u] = reinterpret_cast<uint4*>(z.codes[w] + d * (a.D / 2)) + k;
                v[u] = *reinterpret_cast<const uint4*>(src);
                continue;
            }
            k -= 2 * chunks;
            if (k < 2 * groups) {
                const int w = k >= groups;
                k -= w * groups;
                src = a.pairs[w] + s * groups + k;
                dst[u] = z.pairs[w] + d * groups + k;
            } else if (k == 2 * groups) {
                src = a.weight + s;
                dst[u] = z.weight + d;
            } else {
                src = a.position + s;
                dst[u] = z.position + d;
            }
            v[u].x = *reinterpret_cast<const unsigned*>(src);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!dst[u]) continue;
            if (wide[u]) *reinterpret_cast<uint4*>(dst[u]) = v[u];
            else *reinterpret_cast<unsigned*>(dst[u]) = v[u].x;
        }
    }
}

struct EvictArgs {
    Kv4 a, z;
    int in_place, budget, recent, first;
    int keys;               // capacity of a CTA's key buffer
    int move_here;          // the selecting CTA of a head moves what it listed
    int32_t* counts;        // [B * H] slots to move
    int32_t* lists;         // [B * H][cap]: sources; in place destinations [0, cap / 2), sources from cap / 2 on
};

__device__ __forceinline__ unsigned long long shfl_min(unsigned long long v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const unsigned long long o = __shfl_xor_sync(0xffffffffu, v, d);
        if (o < v) v = o;
    }
    return v;
}

__global__ void __launch_bounds__(1024) kv4_evict_few_kernel(const __grid_constant__ EvictArgs e)
{
    __shared__ unsigned long long buf[32];
    __shared__ int32_t out_s[kEvictFew], from_s[kEvictFew], to_s[kEvictFew];
    __shared__ int moves_s;
    const Kv4& a = e.a;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    wait_for_stream();
    let_next_start();
    const int n = kv4_length(a, b), seen = a.state[b * 4 + kStateSeen];
    const int keep = n < e.budget ? n : e.budget, leave = n - keep;
    const size_t base = ((size_t)b * a.H + h) * a.cap;
    // The next to leave: the smallest key, of equal ones the highest slot; those that have left are skipped.
    int moves = 0;
    for (int r = 0; r < leave; ++r) {
        unsigned long long least = ~0ull;
#pragma unroll 8
        for (int i = tid; i < n; i += blockDim.x) {
            const unsigned u = evict_key(a.weight[base + i], a.position[base + i], seen, e.recent, e.first);
            const unsigned long long v = (unsigned long long)u << 32 | (unsigned)(0x7fffffff - i);
            bool gone = false;
            for (int k = 0; k < r; ++k) gone |= out_s[k] == i;
            if (!gone && v < least) least = v;
        }
        least = shfl_min(least);
        if (lane == 0) buf[warp] = least;
        __syncthreads();
        least = shfl_min(lane < (int)blockDim.x / 32 ? buf[lane] : ~0ull);
        if (tid == 0) out_s[r] = 0x7fffffff - (int)(least & 0xffffffffu);
        __syncthreads();
    }
    if (tid == 0) {
        // free slots below the new length and kept ones above it, both in ascending order
        int hole = -1, at = keep;
        for (;; ++moves) {
            int next = n;
            for (int k = 0; k < leave; ++k)
                if (out_s[k] > hole && out_s[k] < next) next = out_s[k];
            if (next >= keep) break;
            hole = next;
            for (;; ++at) {
                bool left = false;
                for (int k = 0; k < leave; ++k) left |= out_s[k] == at;
                if (!left) break;
            }
            to_s[moves] = hole;
            from_s[moves] = at++;
        }
        moves_s = moves;
    }
    __syncthreads();
    move_slots(a, base, a, base, from_s, to_s, moves_s, tid, blockDim.x);
    if (kv4_last_of_sequence(a, b, gridDim.x)) a.state[b * 4 + kStateLength] = keep;
}

// The new length, by one thread of a sequence's CTAs.  In place it waits until all of them have read the old one; another cache's
// state is read by none, and nothing of the source is written: other calls may be reading it.
__device__ __forceinline__ void set_length(const EvictArgs& e, int b, int keep, int seen)
{
    if (e.in_place ? kv4_last_of_sequence(e.a, b, gridDim.x) : blockIdx.x == 0 && threadIdx.x == 0) {
        e.z.state[b * 4 + kStateLength] = keep;
        e.z.state[b * 4 + kStateSeen] = seen;
    }
}

// Sum over the block's warps before this one, and over all of them.
__device__ __forceinline__ int warps_before(int v, int* buf, int warp, int warps, int* total)
{
    const int lane = threadIdx.x & 31;
    if (lane == 0) buf[warp] = v;
    __syncthreads();
    const int x = lane < warps ? buf[lane] : 0;
    __syncthreads();
    *total = __reduce_add_sync(0xffffffffu, x);
    return __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
}

// Sum of v (the same in all threads of a CTA) over the CTAs before this one, and over all; slots is [kEvictMaxCluster].
__device__ __forceinline__ int ctas_before(int v, int* slots, unsigned rank, unsigned size, int* total)
{
    *total = v;
    if (size == 1) return 0;
    if (threadIdx.x < size) cluster_store(cluster_address(&slots[rank], threadIdx.x), v);
    cluster_sync(size);
    int before = 0, all = 0;
    for (unsigned r = 0; r < size; ++r) {
        all += slots[r];
        before += r < rank ? slots[r] : 0;
    }
    *total = all;
    return before;
}

// The bin, from the top one down, in which the count reaches `want` (1 <= want <= sum of the bins): found = (bin, how many of it
// are wanted, its count).  Called by a whole block of `warps` warps; a warp takes a run of bins, row by row of 32.
__device__ __forceinline__ void find_bin(const unsigned* hist, int want, int warp, int warps, int* buf, int* found)
{
    const int lane = threadIdx.x & 31, run = kEvictBins / warps, first = kEvictBins - (warp + 1) * run;
    int sum = 0;
    for (int k = lane; k < run; k += 32) sum += hist[first + k];
    sum = __reduce_add_sync(0xffffffffu, sum);
    int total;
    int acc = warps_before(sum, buf, warp, warps, &total);
    if (acc < want && want <= acc + sum) {
        for (int k = run - 32;; k -= 32) {
            const int v = hist[first + k + 31 - lane];       // lane 0 has the row's top bin
            int incl = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += u;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, acc + incl >= want);
            if (hit) {
                if (lane == __ffs(hit) - 1) {
                    found[0] = first + k + 31 - lane;
                    found[1] = want - (acc + incl - v);
                    found[2] = v;
                }
                break;
            }
            acc += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    __syncthreads();
}

// Sum of v over the threads before this one in the block, and over all.
__device__ __forceinline__ int threads_before(int v, int* buf, int warp, int warps, int* total)
{
    const int lane = threadIdx.x & 31;
    int incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += u;
    }
    return warps_before(__shfl_sync(0xffffffffu, incl, 31), buf, warp, warps, total) + incl - v;
}

// The selection where a head's slots fit the registers of its CTAs: a thread holds the keys of ITEMS consecutive slots,
// so list order is thread order.  Every CTA of a cluster gets all histograms added up and finds the bins itself.
template <int ITEMS>
__global__ void __launch_bounds__(1024) kv4_select_held_kernel(const __grid_constant__ EvictArgs e)
{
    __shared__ __align__(16) unsigned local[kEvictBins];
    __shared__ __align__(16) unsigned sums[3][kEvictBins + 4];               // per pass; entry kEvictBins: slots that stay for certain
    __shared__ int buf[32], found[4], ties_s[kEvictMaxCluster], movers_s[kEvictMaxCluster], holes_s[kEvictMaxCluster];
    const Kv4& a = e.a;
    const unsigned size = cluster_size(), rank = cluster_rank();
    const int h = blockIdx.x / size, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = warp_number(), warps = blockDim.x >> 5;
    for (int i = tid; i < kEvictBins; i += blockDim.x) local[i] = 0u;
    for (int i = tid; i < 3 * (kEvictBins + 4); i += blockDim.x) (&sums[0][0])[i] = 0u;
    wait_for_stream();
    const int n = kv4_length(a, b), seen = a.state[b * 4 + kStateSeen];
    const int keep = n < e.budget ? n : e.budget;
    const size_t base = ((size_t)b * a.H + h) * a.cap;
    const int share = ((n + (int)size - 1) / (int)size + ITEMS - 1) / ITEMS * ITEMS;
    const int lo = (int)rank * share < n ? (int)rank * share : n, hi = lo + share < n ? lo + share : n;
    const int s0 = lo + tid * ITEMS;                        // this thread's slots; those from hi on are not there
    unsigned key[ITEMS];
    const bool all = keep == n;
    if (!all) {
#pragma unroll
        for (int i = 0; i < ITEMS; i += 4) {
            float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
            int4 p = make_int4(0, 0, 0, 0);
            if (s0 + i < hi) {                              // slots and capacity are multiples of four
                w = *reinterpret_cast<const float4*>(a.weight + base + s0 + i);
                p = *reinterpret_cast<const int4*>(a.position + base + s0 + i);
            }
            key[i] = evict_key(w.x, p.x, seen, e.recent, e.first);
            key[i + 1] = evict_key(w.y, p.y, seen, e.recent, e.first);
            key[i + 2] = evict_key(w.z, p.z, seen, e.recent, e.first);
            key[i + 3] = evict_key(w.w, p.w, seen, e.recent, e.first);
        }
    }
    cluster_sync(size);                                     // the sums are clear everywhere

    // the slots with (key >> shift) > prefix stay, and the first `left` of those with equality
    unsigned prefix = 0u;
    int shift = 0, left = 0;
    bool whole = false;                                     // all of those with equality stay
    if (!all && keep > 0) {
        for (int pass = 0; pass < 3 && !whole; ++pass) {
            shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            const int bits = pass == 2 ? 10 : 11;
            int certain = 0;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const bool in = s0 + i < hi;
                if (key[i] == 0xffffffffu) certain += in;
                else if (in && (pass == 0 || key[i] >> (shift + bits) == prefix)) atomicAdd(&local[(key[i] >> shift) & ((1u << bits) - 1u)], 1u);
            }
            if (pass == 0) {
                certain = __reduce_add_sync(0xffffffffu, certain);
                if (lane == 0 && certain)
                    for (unsigned r = 0; r < size; ++r) cluster_add(cluster_address(&sums[0][kEvictBins], r), certain);
            }
            __syncthreads();
            for (int i = tid * 4; i < kEvictBins; i += blockDim.x * 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(&local[i]);
                const unsigned c[4] = {v.x, v.y, v.z, v.w};
                if ((v.x | v.y | v.z | v.w) == 0u) continue;
                *reinterpret_cast<uint4*>(&local[i]) = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c[k])
                        for (unsigned r = 0; r < size; ++r) cluster_add(cluster_address(&sums[pass][i + k], r), c[k]);
            }
            cluster_sync(size);
            const int want = pass == 0 ? keep - (int)sums[0][kEvictBins] : left;
            if (want <= 0) {
                // only slots that stay for certain do (of more than the budget, with positions that append did not write, the first)
                prefix = 0xffffffffu;
                shift = 0;
                left = keep;
                break;
            }
            find_bin(sums[pass], want, warp, warps, buf, found);
            prefix = pass == 0 ? (unsigned)found[0] : (prefix << bits) | (unsigned)found[0];
            left = found[1];
            whole = found[2] == left;
        }
    }

    int movers = 0;
    if (keep > 0 && !(all && e.in_place)) {
        // bit i of the masks: slot s0 + i
        unsigned ties = 0u, stay = 0u;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool in = s0 + i < hi, sure = key[i] == 0xffffffffu && prefix != 0xffffffffu;
            const bool tie = !all && (key[i] >> shift) == prefix && !sure;
            if (in && tie) ties |= 1u << i;
            if (in && (all || sure || (key[i] >> shift) > prefix)) stay |= 1u << i;
        }
        int ignored;
        if (whole) {
            stay |= ties;
        } else if (!all) {
            int here;
            int rank_of = threads_before(__popc(ties), buf, warp, warps, &here);
            rank_of += ctas_before(here, ties_s, rank, size, &ignored);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (ties >> i & 1u) {
                    if (rank_of < left) stay |= 1u << i;
                    ++rank_of;
                }
        }
        unsigned move = stay, hole = 0u;
        if (e.in_place) {
            const int low = keep - s0 < 0 ? 0 : (keep - s0 > ITEMS ? ITEMS : keep - s0);     // of this thread's slots, those below the new length
            const unsigned below = low >= 32 ? 0xffffffffu : (1u << low) - 1u;
            const int there = hi - s0 < 0 ? 0 : (hi - s0 > ITEMS ? ITEMS : hi - s0);
            const unsigned present = there >= 32 ? 0xffffffffu : (1u << there) - 1u;
            hole = below & present & ~stay;
            move = stay & ~below;
        }
        // one scan for both counts: a CTA has fewer than 2^16 slots
        int here;
        const int at = threads_before(__popc(move) | __popc(hole) << 16, buf, warp, warps, &here);
        int m = (at & 0xffff) + ctas_before(here & 0xffff, movers_s, rank, size, &movers);
        int* list = e.lists + base;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (move >> i & 1u) list[(e.in_place ? a.cap / 2 : 0) + m++] = s0 + i;
        if (e.in_place) {
            int o = (at >> 16) + ctas_before(here >> 16, holes_s, rank, size, &ignored);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (hole >> i & 1u) list[o++] = s0 + i;
        }
    }
    if (tid == 0 && rank == 0) e.counts[b * a.H + h] = movers;
    cluster_sync(size);                                     // the lists are complete, and no CTA ends while another may still write to its shared memory
    let_next_start();
    if (e.move_here) move_slots(a, base, e.z, base, e.lists + base + a.cap / 2, e.lists + base, movers, tid, blockDim.x);
    set_length(e, b, keep, seen);
}

// The selection for heads of any length: keys in shared memory, or read again for each pass.
__global__ void __launch_bounds__(1024) kv4_select_kernel(const __grid_constant__ EvictArgs e)
{
    extern __shared__ __align__(16) unsigned keys[];
    __shared__ unsigned hist[kEvictBins + 1];               // the last: slots that stay for certain
    __shared__ int buf[32], found[4], ties_s[kEvictMaxCluster], movers_s[kEvictMaxCluster], holes_s[kEvictMaxCluster];
    const Kv4& a = e.a;
    const unsigned size = cluster_size(), rank = cluster_rank();
    const int h = blockIdx.x / size, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    wait_for_stream();
    const int n = kv4_length(a, b), seen = a.state[b * 4 + kStateSeen];
    const int keep = n < e.budget ? n : e.budget;
    const size_t base = ((size_t)b * a.H + h) * a.cap;
    const float* weight = a.weight + base;
    const int32_t* position = a.position + base;
    int32_t* list = e.lists + base;
    // this CTA's slots [lo, hi), and of them this warp's [from, to)
    const int share = ((n + (int)size - 1) / (int)size + 31) & ~31;
    const int lo = (int)rank * share < n ? (int)rank * share : n, hi = lo + share < n ? lo + share : n;
    const int per = ((hi - lo + warps - 1) / warps + 31) & ~31;
    const int from = lo + warp * per < hi ? lo + warp * per : hi, to = from + per < hi ? from + per : hi;
    const bool held = hi - lo <= e.keys;
    auto key = [&](int i) { return held ? keys[i - lo] : evict_key(weight[i], position[i], seen, e.recent, e.first); };

    // the slots with (key >> shift) > prefix stay, and the first `left` of those with equality
    unsigned prefix = 0u;
    int shift = 0, left = 0;
    const bool all = keep == n;
    bool whole = false;                                     // all of those with equality stay
    if (!all && keep > 0) {
        for (int pass = 0; pass < 3 && !whole; ++pass) {
            shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            const int bits = pass == 2 ? 10 : 11;
            for (int i = tid; i <= kEvictBins; i += blockDim.x) hist[i] = 0u;
            cluster_sync(size);                             // nobody adds to a histogram that is still being cleared
            if (pass == 0) {
                int certain = 0;
#pragma unroll 4
                for (int i = from + lane; i < to; i += 32) {
                    const unsigned u = evict_key(weight[i], position[i], seen, e.recent, e.first);
                    if (held) keys[i - lo] = u;
                    if (u == 0xffffffffu) ++certain;
                    else atomicAdd(&hist[u >> 21], 1u);
                }
                certain = __reduce_add_sync(0xffffffffu, certain);
                if (lane == 0 && certain) atomicAdd(&hist[kEvictBins], (unsigned)certain);
            } else {
#pragma unroll 4
                for (int i = from + lane; i < to; i += 32) {
                    const unsigned u = key(i);
                    if (u != 0xffffffffu && u >> (shift + bits) == prefix) atomicAdd(&hist[(u >> shift) & ((1u << bits) - 1u)], 1u);
                }
            }
            __syncthreads();
            if (size > 1) {
                if (rank != 0)
                    for (int i = tid; i <= kEvictBins; i += blockDim.x)
                        if (hist[i]) cluster_add(cluster_address(&hist[i], 0), hist[i]);
                cluster_sync(size);
            }
            if (rank == 0) {
                const int want = pass == 0 ? keep - (int)hist[kEvictBins] : left;
                if (want > 0) find_bin(hist, want, warp, warps, buf, found);
                if (tid == 0 && want <= 0) found[1] = 0;     // only slots that stay for certain do
                __syncthreads();
                if (size > 1 && tid < size && tid > 0)
                    for (int k = 0; k < 3; ++k) cluster_store(cluster_address(&found[k], tid), found[k]);
            }
            cluster_sync(size);
            const int bin = found[0], reached = found[1], count = found[2];
            if (pass == 0 && reached == 0) {
                // of more slots that stay for certain than the budget (positions that append did not write): the first ones
                prefix = 0xffffffffu;
                shift = 0;
                left = keep;
                break;
            }
            prefix = pass == 0 ? (unsigned)bin : (prefix << bits) | (unsigned)bin;
            left = reached;
            whole = count == left;
        }
    }

    auto tie = [&](unsigned u) { return (u >> shift) == prefix && (u != 0xffffffffu || prefix == 0xffffffffu); };
    auto over = [&](unsigned u) { return (u >> shift) > prefix || (u == 0xffffffffu && prefix != 0xffffffffu); };
    int movers = 0;
    if (keep > 0 && !(all && e.in_place)) {
        int ties = 0, ignored;
        if (!all && !whole) {
            int c = 0;
            for (int i = from + lane; i < to; i += 32) c += tie(key(i));
            c = __reduce_add_sync(0xffffffffu, c);
            int here;
            ties = warps_before(c, buf, warp, warps, &here);
            ties += ctas_before(here, ties_s, rank, size, &ignored);
        }
        // the lists, in two rounds over the warp's slots: count, then write
        int at[2] = {0, 0};
        for (int round = 0; round < 2; ++round) {
            int seen_ties = ties, m = at[0], o = at[1];
            for (int i0 = from; i0 < to; i0 += 32) {
                const int i = i0 + lane;
                bool stays = i < to;
                if (!all) {
                    const unsigned u = i < to ? key(i) : 0u;
                    const bool eq = i < to && tie(u);
                    bool in = eq;
                    if (!whole) {
                        const unsigned eqs = __ballot_sync(0xffffffffu, eq);
                        in = eq && seen_ties + __popc(eqs & ((1u << lane) - 1u)) < left;
                        seen_ties += __popc(eqs);
                    }
                    stays = i < to && (over(u) || in);
                }
                const bool mover = stays && (!e.in_place || i >= keep), hole = e.in_place && i < to && i < keep && !stays;
                const unsigned ms = __ballot_sync(0xffffffffu, mover), os = __ballot_sync(0xffffffffu, hole);
                if (round) {
                    if (mover) list[(e.in_place ? a.cap / 2 : 0) + m + __popc(ms & ((1u << lane) - 1u))] = i;
                    if (hole) list[o + __popc(os & ((1u << lane) - 1u))] = i;
                }
                m += __popc(ms);
                o += __popc(os);
            }
            if (!round) {
                int here;
                at[0] = warps_before(m, buf, warp, warps, &here);
                at[0] += ctas_before(here, movers_s, rank, size, &movers);
                at[1] = warps_before(o, buf, warp, warps, &here);
                at[1] += ctas_before(here, holes_s, rank, size, &ignored);
            }
        }
    }
    if (tid == 0 && rank == 0) e.counts[b * a.H + h] = movers;
    cluster_sync(size);                                     // no CTA ends while another may still write to its shared memory
    let_next_start();
    set_length(e, b, keep, seen);
}

__global__ void __launch_bounds__(kMoveThreads) kv4_move_kernel(const __grid_constant__ EvictArgs e)
{
    __shared__ int32_t from_s[kMoveSlots], to_s[kMoveSlots];
    const int bh = blockIdx.y, first = blockIdx.x * kMoveSlots, tid = threadIdx.x;
    const size_t base = (size_t)bh * e.a.cap;
    wait_for_stream();
    let_next_start();
    int count = e.counts[bh] - first;
    if (count <= 0) return;
    if (count > kMoveSlots) count = kMoveSlots;
    const int32_t* list = e.lists + base;
    if (tid < count) {
        from_s[tid] = list[(e.in_place ? e.a.cap / 2 : 0) + first + tid];
        to_s[tid] = e.in_place ? list[first + tid] : first + tid;
    }
    __syncthreads();
    move_slots(e.a, base, e.z, (size_t)bh * e.z.cap, from_s, to_s, count, tid, kMoveThreads);
}

static inline size_t evict_lists_at(const Kv4& c) { return ((size_t)c.B * c.H * sizeof(int32_t) + 15) & ~(size_t)15; }

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

coreinfer_status coreinfer_kv4_append(const coreinfer_kv4_cache* cache, const void* k, const void* v,
                                      coreinfer_dtype dtype, int32_t T, int64_t ld_token,
                                      void* k_stored, void* v_stored, void* cuda_stream)
{
    Kv4 c;
    coreinfer_status s = kv4_take(cache, "the", &c);
    if (s != COREINFER_OK) return s;
    if (!dtype_known(dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)dtype);
    if (T < 1) CI_FAIL(COREINFER_ERR_INVALID_ARG, "T must be >= 1");
    if (!k || !v || !aligned16(k) || !aligned16(v)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "k / v NULL or not 16-byte aligned");
    if (ld_token < (int64_t)c.H * c.D || (ld_token * (int64_t)dtype_size(dtype)) % 16 != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "ld_token must cover kv_heads * head_dim elements and be a multiple of 16 bytes");
    if ((k_stored == nullptr) != (v_stored == nullptr) || !aligned16(k_stored) || !aligned16(v_stored))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "k_stored and v_stored come both (16-byte aligned) or neither");
    if ((long long)T * c.H > (1LL << 29)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "T %d: too many tokens for one call", T);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    AppendArgs a;
    a.c = c;
    a.src[0] = k;
    a.src[1] = v;
    a.stored[0] = k_stored;
    a.stored[1] = v_stored;
    a.tokens = T;
    a.rows = T * c.H * 2;
    a.ld = ld_token;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == COREINFER_F32) return pick_append<float>(a, di, st);
    if (dtype == COREINFER_BF16) return pick_append<__nv_bfloat16>(a, di, st);
    return pick_append<__half>(a, di, st);
}

size_t coreinfer_kv4_evict_workspace_bytes(const coreinfer_kv4_cache* src)
{
    Kv4 c;
    if (kv4_take(src, "the source", &c) != COREINFER_OK) return 0;
    return evict_lists_at(c) + (size_t)c.B * c.H * c.cap * sizeof(int32_t);
}

coreinfer_status coreinfer_kv4_evict(const coreinfer_kv4_cache* src, const coreinfer_kv4_cache* dst,
                                     int32_t budget, int32_t recent, int32_t first,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    Kv4 a, z;
    coreinfer_status s = kv4_take(src, "the source", &a);
    if (s != COREINFER_OK || (s = kv4_take(dst, "the destination", &z)) != COREINFER_OK) return s;
    if (!a.weight || !z.weight) CI_FAIL(COREINFER_ERR_INVALID_ARG, "eviction needs caches with weight and position");
    if (budget < 1 || recent < 0 || first < 0 || (long long)recent + first > budget)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "budget %d must be >= 1 and hold recent %d + first %d", budget, recent, first);
    if ((long long)a.B * a.H > 65535) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "batch * kv_heads: at most 65535");
    if (a.B != z.B || a.H != z.H || a.D != z.D || a.G != z.G)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "the two caches differ in batch, kv_heads, head_dim or group");
    int same = 0;
    for (int w = 0; w < 2; ++w) same += (a.codes[w] == z.codes[w]) + (a.pairs[w] == z.pairs[w]);
    same += (a.state == z.state) + (a.weight == z.weight) + (a.position == z.position);
    if (same != 0 && (same != 7 || a.cap != z.cap))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "the two caches share some buffers: all (in place) or none");
    if (z.cap < (budget < a.cap ? budget : a.cap))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "the destination holds %d slots, %d may be kept", z.cap, budget < a.cap ? budget : a.cap);
    if (!workspace || !aligned16(workspace)) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace is NULL or misaligned");
    const size_t need = coreinfer_kv4_evict_workspace_bytes(src);
    if (workspace_bytes < need) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    EvictArgs e;
    e.a = a;
    e.z = z;
    e.in_place = same == 7;
    e.budget = budget;
    e.recent = recent;
    e.first = first;
    e.counts = (int32_t*)workspace;
    e.lists = (int32_t*)((uint8_t*)workspace + evict_lists_at(a));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    // in place no more slots move than there are above the budget
    if (e.in_place && a.cap <= budget) return COREINFER_OK;
    if (e.in_place && a.cap - budget <= kEvictFew) {
        CI_CUDA(launch_overlapped(kv4_evict_few_kernel, dim3(a.H, a.B), dim3(a.cap <= 4096 ? 256 : 1024), 0, st, e));
        return COREINFER_OK;
    }
    // Up to 8 CTAs per head, until 1024 threads hold four slots each, while all of them fit on the GPU at once (1 x 8 heads x
    // 65536 slots: 137 us with one CTA per head, 23 with eight; x 9008: 14.8 with two, 12.7 with four; x 4096: 12.5 with one, 14.4
    // with two).
    int cluster = 1;
    while (cluster < kEvictMaxCluster && a.cap > 4096 * cluster && (long long)a.B * a.H * 2 * cluster <= di.sm_count) cluster *= 2;
    const int per = (a.cap + cluster - 1) / cluster;         // slots per CTA, a multiple of 4 (ITEMS at most divides what follows)
    // in place, what moves comes from above the budget and goes to below it
    const int most = e.in_place ? (a.cap - budget < budget ? a.cap - budget : budget) : (budget < a.cap ? budget : a.cap);
    e.move_here = e.in_place && cluster == 1 && per <= 16384 && most <= kMoveHere;
    if (per <= 16384) {
        // As many threads as there are slots for, while a CTA has an SM to itself (4 x 8 heads x 4096 slots: 14.3 us with 512
        // threads, 12.5 with 1024); where there are more CTAs than SMs, two of 512 threads share one (8 x 32 x 4096: 40 against 46).
        const dim3 held(a.H * cluster, a.B);
        const bool crowded = (long long)a.B * a.H * cluster > di.sm_count;
        if (per <= 1024) CI_CUDA(launch_overlapped(kv4_select_held_kernel<4>, held, dim3(256), 0, st, e, cluster));
        else if (per <= 2048) CI_CUDA(launch_overlapped(kv4_select_held_kernel<4>, held, dim3(512), 0, st, e, cluster));
        else if (per <= 4096 && !crowded) CI_CUDA(launch_overlapped(kv4_select_held_kernel<4>, held, dim3(1024), 0, st, e, cluster));
        else if (per <= 4096) CI_CUDA(launch_overlapped(kv4_select_held_kernel<8>, held, dim3(512), 0, st, e, cluster));
        else if (per <= 8192 && !crowded) CI_CUDA(launch_overlapped(kv4_select_held_kernel<8>, held, dim3(1024), 0, st, e, cluster));
        else if (per <= 8192) CI_CUDA(launch_overlapped(kv4_select_held_kernel<16>, held, dim3(512), 0, st, e, cluster));
        else CI_CUDA(launch_overlapped(kv4_select_held_kernel<16>, held, dim3(1024), 0, st, e, cluster));
    } else {
        const int slots = per + 32;
        e.keys = slots < kEvictKeysMost ? slots : kEvictKeysMost;
        if ((s = allow_smem<kv4_select_kernel>(di, 16384)) != COREINFER_OK) return s;
        CI_CUDA(launch_overlapped(kv4_select_kernel, dim3(a.H * cluster, a.B), dim3(1024), (size_t)e.keys * sizeof(unsigned), st, e, cluster));
    }
    if (e.move_here) return COREINFER_OK;
    CI_CUDA(launch_overlapped(kv4_move_kernel, dim3((most + kMoveSlots - 1) / kMoveSlots, a.B * a.H), dim3(kMoveThreads), 0, st, e));
    return COREINFER_OK;
}

}  // extern "C"
