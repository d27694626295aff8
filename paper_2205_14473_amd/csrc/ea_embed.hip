// ea_embed.hip -- embedding lookup with scaling, and its gradient by sorted
// tokens.
//
// The gradient sorts the ids stably (least significant digits first), cuts the
// sorted order into chunks of equal length and sums each run of equal ids
// inside a chunk; a run that crosses a chunk's end leaves one partial row per
// chunk, joined in order by a second kernel.  The cut depends on the numbers of
// tokens and columns alone, so the order of every sum is fixed by the ids, and
// a token that takes a tenth of the batch costs no more than the others.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_device.hpp"
#include "ea_train.hpp"

namespace ea {

namespace {

constexpr int kRowBlock = 256;

// The row's element quads go to a group of 2^g lanes, 16 to 256; wider rows
// take several slices (or passes) of a group's 4 * 2^g columns.
int group_bits(int64_t dim)
{
    int g = 4;
    while (g < 8 && ((int64_t)4 << g) < dim) ++g;
    return g;
}

__device__ __forceinline__ int64_t id_at(const void* ids, int bits, int64_t i)
{
    return bits == 64 ? ((const int64_t*)ids)[i] : (int64_t)((const int32_t*)ids)[i];
}

// ---- lookup -------------------------------------------------------------------

// x[i] = scale table[ids[i]].  R consecutive tokens a group of lanes: their ids
// first, then a quad of each row.  With more than one the rows written pass the
// caches by, which stay with the table's frequent rows: 65,536 tokens of 1024
// binary32 columns into bfloat16 take 42 us (62 with plain stores, 65 and 81 with
// R = 2 and 8).  Memory bounds it: 270 MB pass the second-level caches, 6.4 TB/s
// (200 MB would be each row once; several XCDs fetch the frequent ones).
template <class T, class X, int R>
__global__ void __launch_bounds__(kRowBlock) lookup_kernel(ea_embed_t c, const T* table, const void* ids, X* x, int gbits)
{
    const int64_t step = ((int64_t)gridDim.x << (8 - gbits)) * R;
    const int lane = threadIdx.x & ((1 << gbits) - 1);
    for (int64_t i = (((int64_t)blockIdx.x << (8 - gbits)) + (threadIdx.x >> gbits)) * R; i < c.tokens; i += step) {
        const T* from[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t id = i + r < c.tokens ? id_at(ids, c.index_bits, i + r) : -1;
            const bool known = id >= 0 && id < c.vocab;
            from[r] = known ? table + id * c.table_stride : nullptr;
        }
        for (int64_t k = lane * 4; k < c.dim; k += (int64_t)4 << gbits) {
            const int n = c.dim - k < 4 ? (int)(c.dim - k) : 4;
            v4f v[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                v[r] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                if (from[r]) v[r] = widen(n == 4 ? load4(from[r] + k) : load_some(from[r] + k, n)) * c.scale;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                X* to = x + (i + r) * c.x_stride + k;
                if (i + r < c.tokens) {
                    if (n != 4)
                        store_some(to, narrow<X>(v[r]), n);
                    else if (R > 1)
                        store4_once(to, narrow<X>(v[r]));
                    else
                        store4(to, narrow<X>(v[r]));
                }
            }
        }
    }
}

// ---- zeros ----------------------------------------------------------------------

// The table's rows as lines of bytes (one line where no elements lie between
// rows), zeroed in units of 16 by workgroups that ride along with the sort's:
// the sort is latency, and the zeros are bandwidth.  (Lines by a division each:
// 50,257 rows of 1,024 binary32 columns in one line 26.3 us, with 32 elements
// between them 26.8, with 5 and so off the 16-byte grid 28.2.)
struct Fill {
    char* base;
    int64_t line, pitch;                 // bytes of a line, and to the next
    int64_t units;                       // 16-byte units of one line
    int64_t begin, end;                  // units of this launch, over all lines
};

template <int THREADS>
__device__ __forceinline__ void fill_zeros(const Fill& f, uint32_t group, uint32_t groups)
{
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
    typedef vec unaligned __attribute__((aligned(2)));
    for (int64_t u = f.begin + (int64_t)group * THREADS + threadIdx.x; u < f.end; u += (int64_t)groups * THREADS) {
        const int64_t line = u < f.units ? 0 : u / f.units, off = (u - line * f.units) * 16;
        char* to = f.base + line * f.pitch + off;
        const int64_t left = f.line - off;
        if (left >= 16)
            *(unaligned*)to = vec{0, 0, 0, 0};
        else
            for (int k = 0; k < (int)left; k += 2) *(uint16_t*)(to + k) = 0;
    }
}

constexpr unsigned kFillGroups = 1024;   // of 1024 threads: 512 and 256 a little slower

__global__ void __launch_bounds__(1024) fill_kernel(Fill f)
{
    fill_zeros<1024>(f, blockIdx.x, gridDim.x);
}

// ---- sort -----------------------------------------------------------------------

constexpr int kSortBlock = 1024;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kMostBits = 9;             // of one pass's digit
constexpr int kMostValues = 1 << kMostBits;
constexpr int kRounds = 4;               // items a lane holds, at most
constexpr int64_t kMostTile = kSortBlock * kRounds;
constexpr int64_t kMidTile = kSortBlock * 2;
constexpr int64_t kLeastTile = kSortBlock;
constexpr int64_t kFewTiles = 128;       // whose counts every workgroup of a scatter adds up itself
constexpr int kTilesAhead = 16;          // tiles' counts a thread loads ahead
static_assert(kSortBlock >= 2 * kMostValues, "a digit has threads to share its tiles");

struct SortPlan {
    int64_t n, tiles;
    int tile;                            // items of one workgroup
    int passes, bits;                    // digit width of each pass
};

SortPlan sort_plan(const ea_embed_t& c)
{
    SortPlan p;
    p.n = c.tokens;
    // the smallest tiles that leave few of them: 32,768 ids 56 us with 1,024 a tile, 60 with 2,048
    p.tile = (int)(c.tokens <= kLeastTile * kFewTiles ? kLeastTile : c.tokens <= kMidTile * kFewTiles ? kMidTile : kMostTile);
    p.tiles = (c.tokens + p.tile - 1) / p.tile;
    int need = 1;
    while (c.vocab >> need) ++need;      // keys are 0 to vocab
    p.passes = (need + kMostBits - 1) / kMostBits;
    p.bits = (need + p.passes - 1) / p.passes;
    return p;
}

// Items to sort: the ids themselves before the first pass, then (key, position).
struct Items {
    const void* ids;                     // first pass; null afterwards
    const uint32_t* keys;
    const uint32_t* at;
    int index_bits;
    int64_t vocab, padding;
};

__device__ __forceinline__ uint32_t key_of(const Items& t, int64_t i)
{
    if (!t.ids) return t.keys[i];
    const int64_t id = id_at(t.ids, t.index_bits, i);
    return id >= 0 && id < t.vocab && id != t.padding ? (uint32_t)id : (uint32_t)t.vocab;
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A lane's place among its wave's items of one digit: `count` holds the digits'
// running counts, which move on by the 64 lanes' items.
template <class C>
__device__ __forceinline__ uint32_t take_place(C* count, uint32_t digit, int bits, bool here)
{
    uint64_t same = __ballot(here);
    for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? ones : ~ones;
    }
    const uint64_t lower = same & ((1ull << lane_id()) - 1);
    const uint32_t first = here ? count[digit] : 0;
    wave_sync();
    if (here && !lower) count[digit] = (C)(first + (uint32_t)__popcll(same));
    wave_sync();
    return first + (uint32_t)__popcll(lower);
}

// Exclusive sum over the workgroup's threads.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* sums)
{
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    uint32_t upto = x;
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t k = __shfl_up(upto, d);
        upto += lane >= d ? k : 0;
    }
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    uint32_t base = upto - x;
    for (int w = 0; w < wave; ++w) base += sums[w];
    return base;
}

// Offsets of every wave's items of every digit, in place of its counts: `base`
// is the first item of thread v's digit.
template <class C>
__device__ __forceinline__ void place_waves(C (*place)[kMostValues], int values, uint32_t base)
{
    if ((int)threadIdx.x < values) {
        uint32_t k[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) k[w] = place[w][threadIdx.x];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            place[w][threadIdx.x] = (C)base;
            base += k[w];
        }
    }
    __syncthreads();
}

template <class C>
__device__ __forceinline__ void no_places(C (*place)[kMostValues], int bits)
{
    for (int k = threadIdx.x; k < kSortWaves << bits; k += kSortBlock) place[k >> bits][k & ((1 << bits) - 1)] = 0;
}

// Tokens that one workgroup sorts in its registers and LDS, every pass in one
// launch; the other workgroups zero the table.  64 ids 6 us, 4,096 about 12, both
// under the 15 us that zeroing 32,000 rows of 768 takes.  (Twice as many
// items a lane, for 8,192 ids, took as long as the launches below.)
__global__ void __launch_bounds__(kSortBlock) sort_one_kernel(Items t, SortPlan p, uint32_t* keys, uint32_t* at, Fill f)
{
    __shared__ uint16_t place[kSortWaves][kMostValues];
    __shared__ uint32_t skey[kMostTile];  // and sum_before's sums, while the registers hold the keys
    __shared__ uint16_t sat[kMostTile];
    if (blockIdx.x > 0) {
        fill_zeros<kSortBlock>(f, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const int values = 1 << p.bits, wave = threadIdx.x / kWave, lane = lane_id(), n = (int)p.n;
    const int rounds = (n + kSortBlock - 1) / kSortBlock, begin = wave * rounds * kWave + lane;
    uint32_t key[kRounds], from[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = begin + r * kWave;
        from[r] = (uint32_t)i;
        key[r] = r < rounds && i < n ? key_of(t, i) : 0;
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * p.bits;
        no_places(place, p.bits);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            if (r < rounds)
                rank[r] = take_place(place[wave], (key[r] >> shift) & (values - 1), p.bits, begin + r * kWave < n);
        __syncthreads();
        uint32_t all = 0;
        if ((int)threadIdx.x < values) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) all += place[w][threadIdx.x];
        }
        place_waves(place, values, sum_before(all, skey));
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            if (r < rounds && begin + r * kWave < n) {
                const uint32_t to = place[wave][(key[r] >> shift) & (values - 1)] + rank[r];
                skey[to] = key[r];
                sat[to] = (uint16_t)from[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = begin + r * kWave;
            if (r < rounds && i < n) {
                key[r] = skey[i];
                from[r] = sat[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = begin + r * kWave;
        if (r < rounds && i < n) {
            keys[i] = key[r];
            at[i] = from[r];
        }
    }
}

constexpr int kFewTokens = 512;          // that one workgroup ranks by comparing all with all

// So few that comparing each with all is the shortest: 2^bits threads a token,
// a share of the others each.  256 ids 3 us (in digits 6), 512 4.5; the work grows
// with the square (1,024 took 45).
__global__ void __launch_bounds__(kSortBlock) rank_kernel(Items t, int n, int bits, uint32_t* keys, uint32_t* at, Fill f)
{
    __shared__ uint4 all[kFewTokens / 4];
    if (blockIdx.x > 0) {
        fill_zeros<kSortBlock>(f, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const int i = threadIdx.x >> bits, shares = 1 << bits, share = threadIdx.x & (shares - 1), own = i / 4;
    const uint32_t key = i < n ? key_of(t, i) : 0xFFFFFFFFu;
    if (share == 0 && i < kFewTokens) ((uint32_t*)all)[i] = key;
    __syncthreads();
    int rank = 0;
#pragma unroll 4
    for (int q = share; q < (n + 3) / 4; q += shares) {
        const uint4 x = all[q];
        const uint32_t above = q < own ? key + 1 : key;    // equal ids before this one come first
        rank += (x.x < above) + (x.y < above) + (x.z < above) + (x.w < above);
    }
    if (share == 0 && i < n) {                             // and those of the same four
        const uint4 x = all[own];
        rank += (i % 4 > 0 && x.x == key) + (i % 4 > 1 && x.y == key) + (i % 4 > 2 && x.z == key);
    }
    for (int d = 1; d < shares; d *= 2) rank += __shfl_xor(rank, d);
    if (share == 0 && i < n) {
        keys[rank] = key;
        at[rank] = (uint32_t)i;
    }
}

// Larger batches: the digits of each tile counted, then the tile's items put in place.
__global__ void __launch_bounds__(kSortBlock) digits_kernel(Items t, SortPlan p, int shift, uint32_t* counts)
{
    __shared__ uint32_t count[kMostValues];
    const int values = 1 << p.bits;
    const int64_t begin = (int64_t)blockIdx.x * p.tile + threadIdx.x;
    uint32_t key[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = begin + r * kSortBlock;
        key[r] = r * kSortBlock < p.tile && i < p.n ? key_of(t, i) : 0;
    }
    if ((int)threadIdx.x < values) count[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r * kSortBlock < p.tile && begin + r * kSortBlock < p.n)
            atomicAdd(&count[(key[r] >> shift) & (values - 1)], 1u);
    __syncthreads();
    if ((int)threadIdx.x < values) counts[(int64_t)blockIdx.x * values + threadIdx.x] = count[threadIdx.x];
}

// Many tiles: workgroup v turns digit v's counts into sums over the tiles
// before each, and their total into the row after the last tile's.
__global__ void __launch_bounds__(kSortBlock) prefix_kernel(SortPlan p, uint32_t* counts)
{
    __shared__ uint32_t sums[kSortWaves];
    const int64_t values = (int64_t)1 << p.bits;
    uint32_t* c = counts + blockIdx.x;
    uint32_t base = 0;
    for (int64_t b = 0; b < p.tiles; b += kSortBlock) {
        const int64_t tile = b + threadIdx.x;
        const uint32_t k = tile < p.tiles ? c[tile * values] : 0;
        const uint32_t upto = sum_before(k, sums);
        if (tile < p.tiles) c[tile * values] = base + upto;
        uint32_t all = 0;
        for (int w = 0; w < kSortWaves; ++w) all += sums[w];
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) c[p.tiles * values] = base;
}

// Each wave owns a run of its tile's items and ranks them among its own, 64 at
// a time, in order; waves, tiles and digits before then add their counts.
// Latency bounds it, a dozen dependent trips: 7.5 us for 8,192 to 131,072 ids, 16
// with 103 MB of zeros written beside it (13 by themselves).
__global__ void __launch_bounds__(kSortBlock) scatter_kernel(Items t, SortPlan p, int shift, const uint32_t* counts,
                                                             uint32_t* keys, uint32_t* at, Fill f)
{
    __shared__ uint32_t place[kSortWaves][kMostValues];
    __shared__ uint32_t totals[2][kMostValues];
    __shared__ uint32_t sums[kSortWaves];
    if (blockIdx.x >= p.tiles) {
        fill_zeros<kSortBlock>(f, blockIdx.x - (uint32_t)p.tiles, gridDim.x - (uint32_t)p.tiles);
        return;
    }
    const int values = 1 << p.bits, wave = threadIdx.x / kWave, rounds = p.tile / kSortBlock;
    const int64_t begin = (int64_t)blockIdx.x * p.tile + wave * rounds * kWave + lane_id();
    uint32_t key[kRounds], from[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = begin + r * kWave;
        const bool here = r < rounds && i < p.n;
        key[r] = here ? key_of(t, i) : 0;
        from[r] = here && !t.ids ? t.at[i] : (uint32_t)i;
    }

    // items with each digit in all tiles, and in the tiles before this one: the
    // tiles' counts shared out among the threads of a digit
    const uint32_t v = threadIdx.x & (values - 1);
    uint32_t some = 0, some_before = 0;
    if (p.tiles > kFewTiles) {
        if ((int)threadIdx.x < values) {
            some = counts[p.tiles * values + v];
            some_before = counts[(int64_t)blockIdx.x * values + v];
        }
    } else {
        const int shares = kSortBlock >> p.bits, tiles = (int)p.tiles;
        for (int b = threadIdx.x >> p.bits; b < tiles; b += shares * kTilesAhead) {
            uint32_t k[kTilesAhead];
#pragma unroll
            for (int r = 0; r < kTilesAhead; ++r) {
                const int tile = b + r * shares;
                k[r] = counts[(tile < tiles ? tile : b) * values + v];
            }
#pragma unroll
            for (int r = 0; r < kTilesAhead; ++r) {
                const int tile = b + r * shares;
                some += tile < tiles ? k[r] : 0;
                some_before += tile < (int)blockIdx.x ? k[r] : 0;
            }
        }
    }
    no_places(place, p.bits);
    (&totals[0][0])[threadIdx.x] = 0;
    __syncthreads();
    atomicAdd(&totals[0][v], some);
    atomicAdd(&totals[1][v], some_before);
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds)
            rank[r] = take_place(place[wave], (key[r] >> shift) & (values - 1), p.bits, begin + r * kWave < p.n);
    __syncthreads();
    const bool one = (int)threadIdx.x < values;
    const uint32_t base = sum_before(one ? totals[0][v] : 0, sums);
    place_waves(place, values, base + (one ? totals[1][v] : 0));
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds && begin + r * kWave < p.n) {
            const uint32_t to = place[wave][(key[r] >> shift) & (values - 1)] + rank[r];
            keys[to] = key[r];
            at[to] = from[r];
        }
}

// ---- sums -------------------------------------------------------------------------

struct SumArgs {
    int64_t n, chunk, chunks, vocab, dim, table_stride, x_stride;
    const uint32_t* keys;
    const uint32_t* at;
    float* part;                         // [chunks][2][dim rounded up to 4]
    int64_t part_row;
    float scale;
    int gbits, accumulate;
};

constexpr int kMostChunk = kWave;        // a lane for each position of a chunk
constexpr int kAhead = 8;                // rows a lane loads ahead

template <class T>
__device__ __forceinline__ void finish_row(const SumArgs& a, T* table, uint32_t key, int64_t col, int n, v4f sum)
{
    T* to = table + (int64_t)key * a.table_stride + col;
    v4f v = sum * a.scale;
    if (a.accumulate) v = v + widen(n == 4 ? load4(to) : load_some(to, n));
    if (n == 4)
        store4(to, narrow<T>(v));
    else
        store_some(to, narrow<T>(v), n);
}

// A group of lanes sums one chunk of the sorted order over its slice of the
// columns.  A row is finished here where its run lies within the chunk; a run
// that came from the chunk before goes to partial row 0, one that goes on in
// the chunk after to partial row 1.  Groups are whole waves: a lane holds one
// position's key and row, from which the wave takes the next rows' addresses and
// the ends of the runs without a branch of its own.  (Rows of up to 128 columns
// leave lanes idle; with several groups a wave, each lane for itself, 131,072
// rows of 128 binary32 columns took 105 us in all, against 57.)  HBM bounds it: 131,072
// rows of 1024 bfloat16 columns 71 us, 5.3 TB/s with the rows and partial rows
// written (95 us with dx through the caches, which the sums' rows then leave).
template <class T, class X>
__global__ void __launch_bounds__(kRowBlock) sum_kernel(SumArgs a, const X* dx, T* table)
{
    const int lane = lane_id();
    const int64_t c = ((int64_t)blockIdx.x << (8 - a.gbits)) +
                      __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> a.gbits));
    const int64_t col = (((int64_t)blockIdx.y << a.gbits) + (threadIdx.x & ((1 << a.gbits) - 1))) * 4;
    if (c >= a.chunks) return;
    const int64_t begin = c * a.chunk;
    const int count = (int)(a.n - begin < a.chunk ? a.n - begin : a.chunk);
    // lane l: position l; the keys beside the chunk say whether its first and last runs go on there
    const uint32_t none = 0xFFFFFFFFu;
    const int64_t mine = begin + (lane < count ? lane : count - 1);
    const uint32_t key = a.keys[mine], at = a.at[mine];
    const uint32_t last_key = begin > 0 ? a.keys[begin - 1] : none;
    const uint32_t next_key = begin + count < a.n ? a.keys[begin + count] : none;
    uint32_t left = __shfl_up(key, 1);
    if (lane == 0) left = last_key;
    const uint64_t starts = __ballot(lane < count && key != left);
    const int used = __popcll(__ballot(lane < count && key < a.vocab));   // the others sort last
    if (used == 0) return;
    const int n = a.dim - col >= 4 ? 4 : a.dim > col ? (int)(a.dim - col) : 0;
    float* part = a.part + c * 2 * a.part_row + col;
    bool open = !(starts & 1);                             // the first run began before this chunk
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < used; k += kAhead) {
        typename Quad<X>::vec x[kAhead];
#pragma unroll
        for (int r = 0; r < kAhead; ++r) {
            const int i = k + r < used ? k + r : used - 1;
            const X* from = dx + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, i) * a.x_stride + col;
            x[r] = n == 4 ? load4_once(from) : load_some(from, n);
        }
#pragma unroll
        for (int r = 0; r < kAhead; ++r) {
            if (k + r >= used) break;
            if (k + r > 0 && ((starts >> (k + r)) & 1)) {
                if (n > 0) {
                    if (open)
                        store4(part, sum);
                    else
                        finish_row(a, table, (uint32_t)__builtin_amdgcn_readlane((int)key, k + r - 1), col, n, sum);
                }
                open = false;
                sum = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
            sum = sum + widen(x[r]);
        }
    }
    const uint32_t end_key = (uint32_t)__builtin_amdgcn_readlane((int)key, used - 1);
    if (n == 0) return;
    if (open)
        store4(part, sum);
    else if (used == count && next_key == end_key)
        store4(part + a.part_row, sum);
    else
        finish_row(a, table, end_key, col, n, sum);
}

// Few tokens: a workgroup a position of the sorted order, of which those where a
// run begins sum the run; no row is split and nothing is left to join.
template <class T, class X>
__global__ void __launch_bounds__(kRowBlock) sum_runs_kernel(SumArgs a, const X* dx, T* table)
{
    const int lane = lane_id(), i = blockIdx.x, count = (int)a.n;
    const int64_t col = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * 4;
    const int n = a.dim - col >= 4 ? 4 : a.dim > col ? (int)(a.dim - col) : 0;
    const uint32_t key = a.keys[i], before = a.keys[i > 0 ? i - 1 : 0];
    int from = i, mine = from + lane < count ? from + lane : count - 1;
    uint32_t others = a.keys[mine], at = a.at[mine];
    if ((key >= a.vocab) | ((i > 0) & (before == key))) return;
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (;;) {
        const int run = __popcll(__ballot(from + lane < count && others == key));
        for (int k = 0; k < run; k += kAhead) {
            typename Quad<X>::vec x[kAhead];
#pragma unroll
            for (int r = 0; r < kAhead; ++r) {
                const int p = k + r < run ? k + r : run - 1;
                const X* row = dx + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, p) * a.x_stride + col;
                x[r] = n == 4 ? load4_once(row) : load_some(row, n);
            }
#pragma unroll
            for (int r = 0; r < kAhead; ++r)
                if (k + r < run) sum = sum + widen(x[r]);
        }
        from += kWave;
        if (run < kWave || from >= count) break;
        mine = from + lane < count ? from + lane : count - 1;
        others = a.keys[mine];
        at = a.at[mine];
    }
    if (n > 0) finish_row(a, table, key, col, n, sum);
}

constexpr int kJoinWaves = kRowBlock / kWave;
constexpr int kJoinCols = kWave * 4;

// The runs that cross chunks: the workgroup of the chunk in which one begins
// adds up its partial rows, a quarter of them to each wave, in an order that
// their number fixes.  Latency: 4 us for 256 chunks, 12 for 2,048 and a token
// with a tenth of them.
template <class T>
__global__ void __launch_bounds__(kRowBlock) join_kernel(SumArgs a, T* table)
{
    __shared__ v4f sums[kJoinWaves][kWave];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int64_t c = blockIdx.x, begin = c * a.chunk, end = begin + a.chunk;
    if (end >= a.n) return;
    // all keys at once, the next 64 chunks' first ones among them: most workgroups end here
    const uint32_t key = a.keys[end - 1], next = a.keys[end], head = a.keys[begin];
    const uint32_t before = a.keys[begin > 0 ? begin - 1 : 0];
    int64_t rows = a.chunks - 1 - c, range = 0;
    const uint32_t heads = a.keys[end + (lane < rows ? lane : 0) * a.chunk];
    if ((key >= a.vocab) | (next != key)) return;                                  // ends here
    if ((begin > 0) & (head == key) & (before == key)) return;                     // began before
    // the chunks after this one whose first key is still `key`
    {
        const int hits = __popcll(__ballot(lane < rows && heads == key));
        if (hits == kWave) range = rows - kWave;
        rows = hits;
    }
    while (range > 0) {                                                            // more: a 64-way search
        const int64_t step = (range + kWave - 1) / kWave, probe = lane * step;
        const bool still = probe < range && a.keys[end + (rows + probe) * a.chunk] == key;
        const int hits = __popcll(__ballot(still));
        if (hits == 0) break;
        const int64_t known = (hits - 1) * step + 1;
        range = range - known < step - 1 ? range - known : step - 1;
        rows += known;
    }
    const int64_t col = (int64_t)blockIdx.y * kJoinCols + lane * 4;
    const int64_t each = (rows + kJoinWaves - 1) / kJoinWaves;
    const int64_t from = wave * each, upto = from + each < rows ? from + each : rows;
    const float* part = a.part + (c + 1) * 2 * a.part_row + col;
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < a.dim) {
        for (int64_t k = from; k < upto; k += 2 * kAhead) {
            v4f x[2 * kAhead];
#pragma unroll
            for (int r = 0; r < 2 * kAhead; ++r)
                x[r] = load4(part + (k + r < upto ? k + r : upto - 1) * 2 * a.part_row);
#pragma unroll
            for (int r = 0; r < 2 * kAhead; ++r)
                if (k + r < upto) sum = sum + x[r];
        }
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && col < a.dim) {
        sum = load4(part - a.part_row);                                            // this chunk's
        for (int w = 0; w < kJoinWaves; ++w) sum = sum + sums[w][lane];
        finish_row(a, table, key, col, a.dim - col < 4 ? (int)(a.dim - col) : 4, sum);
    }
}

struct GradPlan {
    SortPlan sort;
    int64_t chunk, chunks, part_row;
    int64_t off_keys[2], off_at[2], off_counts, off_part, bytes;
};

int64_t align16(int64_t x)
{
    return (x + 15) / 16 * 16;
}

constexpr int64_t kEnoughWaves = 4096;   // 16 for each CU (8192: 16,384 tokens 49 us against 46)
constexpr int64_t kLeastChunk = 8;

// Positions of a chunk: 64, or fewer where that leaves CUs without waves.
int64_t chunk_of(int64_t tokens, int64_t dim)
{
    const int64_t waves = (dim + kJoinCols - 1) / kJoinCols;
    int64_t chunk = kMostChunk;
    while (chunk > kLeastChunk && tokens / chunk * waves < kEnoughWaves) chunk /= 2;
    return chunk;
}

GradPlan grad_plan(const ea_embed_t& c)
{
    GradPlan p{};
    if (c.tokens == 0) return p;
    p.sort = sort_plan(c);
    p.chunk = chunk_of(c.tokens, c.dim);
    p.chunks = (c.tokens + p.chunk - 1) / p.chunk;
    p.part_row = (c.dim + 3) / 4 * 4;
    int64_t off = 0;
    for (int k = 0; k < 2; ++k) {
        p.off_keys[k] = off;
        off += align16(c.tokens * 4);
        p.off_at[k] = off;
        off += align16(c.tokens * 4);
    }
    p.off_counts = off;
    off += align16((p.sort.tiles + 1) * ((int64_t)4 << p.sort.bits));
    p.off_part = off;
    off += p.chunks * 2 * p.part_row * 4;
    p.bytes = off;
    return p;
}

// Workgroups for `rows` rows, one group of lanes each; the kernel loops over the rest.
unsigned row_groups(int64_t rows, int gbits)
{
    const int64_t per = (int64_t)1 << (8 - gbits), blocks = (rows + per - 1) / per;
    return (unsigned)(blocks < (1 << 22) ? blocks : (1 << 22));
}

// The part of the zeros that goes with launch k of `of`.
Fill fill_part(Fill f, int64_t units, int k, int of)
{
    f.begin = units / of * k;
    f.end = k == of - 1 ? units : units / of * (k + 1);
    return f;
}

template <class T, class X>
hipError_t start_grad(const ea_embed_t& c, const GradPlan& p, const void* ids, const X* dx, T* table, bool accumulate,
                      char* ws, hipStream_t s)
{
    Fill f{};
    f.base = (char*)table;
    f.line = c.dim * (int64_t)sizeof(T);
    f.pitch = c.table_stride * (int64_t)sizeof(T);
    int64_t lines = accumulate ? 0 : c.vocab;
    if (f.line == f.pitch || lines == 1) {
        f.line = lines * f.line;
        lines = lines > 0 ? 1 : 0;
    }
    f.units = (f.line + 15) / 16;
    const int64_t units = f.units * lines;
    const unsigned groups = units == 0 ? 0 : (unsigned)(units / kSortBlock < kFillGroups ? units / kSortBlock + 1 : kFillGroups);
    if (c.tokens == 0) {
        if (groups == 0) return hipSuccess;
        hipLaunchKernelGGL(fill_kernel, dim3(groups), dim3(kSortBlock), 0, s, fill_part(f, units, 0, 1));
        return hipGetLastError();
    }
    Items t{ids, nullptr, nullptr, c.index_bits, c.vocab, c.padding};
    uint32_t* counts = (uint32_t*)(ws + p.off_counts);
    const auto keys = [&](int k) { return (uint32_t*)(ws + p.off_keys[k & 1]); };
    const auto at = [&](int k) { return (uint32_t*)(ws + p.off_at[k & 1]); };
    if (c.tokens <= kFewTokens) {
        int bits = 0;
        while (bits < 3 && c.tokens << (bits + 1) <= kSortBlock) ++bits;
        hipLaunchKernelGGL(rank_kernel, dim3(1 + groups), dim3(kSortBlock), 0, s, t, (int)c.tokens, bits, keys(0), at(0),
                           fill_part(f, units, 0, 1));
        t.keys = keys(0);
        t.at = at(0);
    } else if (c.tokens <= kMostTile) {
        hipLaunchKernelGGL(sort_one_kernel, dim3(1 + groups), dim3(kSortBlock), 0, s, t, p.sort, keys(0), at(0),
                           fill_part(f, units, 0, 1));
        t.keys = keys(0);
        t.at = at(0);
    } else {
        const unsigned tiles = (unsigned)p.sort.tiles;
        for (int k = 0; k < p.sort.passes; ++k) {
            const int shift = k * p.sort.bits;
            hipLaunchKernelGGL(digits_kernel, dim3(tiles), dim3(kSortBlock), 0, s, t, p.sort, shift, counts);
            if (p.sort.tiles > kFewTiles)
                hipLaunchKernelGGL(prefix_kernel, dim3(1u << p.sort.bits), dim3(kSortBlock), 0, s, p.sort, counts);
            hipLaunchKernelGGL(scatter_kernel, dim3(tiles + groups), dim3(kSortBlock), 0, s, t, p.sort, shift, counts,
                               keys(k), at(k), fill_part(f, units, k, p.sort.passes));
            t.ids = nullptr;
            t.keys = keys(k);
            t.at = at(k);
        }
    }
    SumArgs a{};
    a.n = c.tokens;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.vocab = c.vocab;
    a.dim = c.dim;
    a.table_stride = c.table_stride;
    a.x_stride = c.x_stride;
    a.keys = t.keys;
    a.at = t.at;
    a.part = (float*)(ws + p.off_part);
    a.part_row = p.part_row;
    a.scale = c.scale;
    a.gbits = c.dim <= kJoinCols ? 6 : group_bits(c.dim);   // whole waves, also of narrow rows
    a.accumulate = accumulate ? 1 : 0;
    if (c.tokens <= kFewTokens) {
        const int64_t waves = c.dim > 3 * kJoinCols ? 4 : (c.dim + kJoinCols - 1) / kJoinCols, cols = waves * kJoinCols;
        hipLaunchKernelGGL((sum_runs_kernel<T, X>), dim3((unsigned)c.tokens, (unsigned)((c.dim + cols - 1) / cols)),
                           dim3((unsigned)(waves * kWave)), 0, s, a, dx, table);
        return hipGetLastError();
    }
    const int64_t per = (int64_t)1 << (8 - a.gbits);
    const dim3 grid((unsigned)((p.chunks + per - 1) / per),
                    (unsigned)((c.dim + ((int64_t)4 << a.gbits) - 1) >> (2 + a.gbits)));
    hipLaunchKernelGGL((sum_kernel<T, X>), grid, dim3(kRowBlock), 0, s, a, dx, table);
    if (p.chunks > 1)
        hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)(p.chunks - 1), (unsigned)((c.dim + kJoinCols - 1) / kJoinCols)),
                           dim3(kRowBlock), 0, s, a, table);
    return hipGetLastError();
}

// A group of lanes takes four tokens where they fill the GPU: from 3M elements and 4,096 tokens on; otherwise
// one.  Binary32, us on the GPU for one and four: 8,192 tokens of 64 columns 2.2 and 3.1, 32,768 3.6 and 4.0,
// 4,096 of 256 2.7 and 3.3, of 768 4.9 and 4.5, 8,192 of 1,024 11.5 and 10.5, 65,536 97 and 76; few and wide,
// 1,024 of 4,096 5.4 and 6.8, 4,096 of them 21.1 and 21.2.  The 16-bit types cross between 2.1M and 4.2M alike.
constexpr int64_t kFourElements = 3 << 20;
constexpr int64_t kFourTokens = 4096;

// f(table element, row element) with the types that c names.
template <class F, class T>
hipError_t with_x(const ea_embed_t& c, T t, const F& f)
{
    if (c.x_type == EA_F32) return f(t, float());
    if (c.x_type == EA_BF16) return f(t, bf16());
    return f(t, f16());
}

template <class F>
hipError_t with_types(const ea_embed_t& c, const F& f)
{
    if (c.table_type == EA_F32) return with_x(c, float(), f);
    if (c.table_type == EA_BF16) return with_x(c, bf16(), f);
    return with_x(c, f16(), f);
}

}  // namespace

hipError_t launch_embed_lookup(const ea_embed_t& c, const void* table, const void* ids, void* x, hipStream_t s)
{
    if (c.tokens == 0) return hipSuccess;
    const int gbits = group_bits(c.dim);
    return with_types(c, [&](auto t, auto e) {
        using T = decltype(t);
        using X = decltype(e);
        if (c.tokens < kFourTokens || c.tokens * c.dim < kFourElements)
            hipLaunchKernelGGL((lookup_kernel<T, X, 1>), dim3(row_groups(c.tokens, gbits)), dim3(kRowBlock), 0, s, c,
                               (const T*)table, ids, (X*)x, gbits);
        else
            hipLaunchKernelGGL((lookup_kernel<T, X, 4>), dim3(row_groups((c.tokens + 3) / 4, gbits)), dim3(kRowBlock), 0, s,
                               c, (const T*)table, ids, (X*)x, gbits);
        return hipGetLastError();
    });
}

int64_t embed_workspace_bytes(const ea_embed_t& c)
{
    return grad_plan(c).bytes;
}

hipError_t launch_embed_grad(const ea_embed_t& c, const void* ids, const void* dx, void* dtable, bool accumulate,
                             void* workspace, hipStream_t s)
{
    const GradPlan p = grad_plan(c);
    return with_types(c, [&](auto t, auto e) {
        using T = decltype(t);
        using X = decltype(e);
        return start_grad<T, X>(c, p, ids, (const X*)dx, (T*)dtable, accumulate, (char*)workspace, s);
    });
}

}  // namespace ea
