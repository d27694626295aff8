// ea_embed.hip -- embedding lookup with scaling, and its gradient by sorted
// tokens.
//
// The gradient sorts the ids stably (least significant digits first), cuts the
// sorted order into chunks of equal length and sums each run of equal ids
// inside a chunk; a run that crosses a chunk's end leaves one partial row per
// chunk, joined in order by a second kernel.  The cut depends on the number
// of tokens alone, so the order of every sum is fixed by the ids, and a
// token that takes a tenth of the batch costs no more than the others.
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

template <class T, class X>
__global__ void __launch_bounds__(kRowBlock) lookup_kernel(ea_embed_t c, const T* table, const void* ids, X* x, int gbits)
{
    const int64_t rows = (int64_t)gridDim.x << (8 - gbits);
    const int lane = threadIdx.x & ((1 << gbits) - 1);
    for (int64_t i = ((int64_t)blockIdx.x << (8 - gbits)) + (threadIdx.x >> gbits); i < c.tokens; i += rows) {
        const int64_t id = id_at(ids, c.index_bits, i);
        const bool known = id >= 0 && id < c.vocab;
        const T* from = table + (known ? id : 0) * c.table_stride;
        X* to = x + i * c.x_stride;
        for (int64_t k = lane * 4; k < c.dim; k += (int64_t)4 << gbits) {
            const int n = c.dim - k < 4 ? (int)(c.dim - k) : 4;
            v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
            if (known) v = widen(n == 4 ? load4(from + k) : load_some(from + k, n)) * c.scale;
            if (n == 4)
                store4(to + k, narrow<X>(v));
            else
                store_some(to + k, narrow<X>(v), n);
        }
    }
}

// ---- sort -----------------------------------------------------------------------

constexpr int kSortBlock = 512;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kMostBits = 9;             // of one pass's digit: a thread for each value
constexpr int64_t kLeastTile = 2048;     // items of one workgroup
constexpr int64_t kMostTiles = 128;

struct SortPlan {
    int64_t n, tile, tiles;
    int passes, bits;                    // digit width of each pass
};

SortPlan sort_plan(const ea_embed_t& c)
{
    SortPlan p;
    p.n = c.tokens;
    p.tile = (c.tokens + kMostTiles - 1) / kMostTiles;
    p.tile = (p.tile + kSortBlock - 1) / kSortBlock * kSortBlock;
    if (p.tile < kLeastTile) p.tile = kLeastTile;
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

__global__ void __launch_bounds__(kSortBlock) digits_kernel(Items t, SortPlan p, int shift, uint32_t* counts)
{
    __shared__ uint32_t count[1 << kMostBits];
    const int values = 1 << p.bits;
    if ((int)threadIdx.x < values) count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * p.tile, end = begin + p.tile < p.n ? begin + p.tile : p.n;
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortBlock)
        atomicAdd(&count[(key_of(t, i) >> shift) & (values - 1)], 1u);
    __syncthreads();
    if ((int)threadIdx.x < values) counts[(int64_t)blockIdx.x * values + threadIdx.x] = count[threadIdx.x];
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Each wave owns a run of its tile's items.  Their digits are counted once to
// place the waves, then walked in order, 64 at a time: a lane's place is its
// digit's running count plus the equal digits in lower lanes.
__global__ void __launch_bounds__(kSortBlock) scatter_kernel(Items t, SortPlan p, int shift, const uint32_t* counts,
                                                             uint32_t* keys, uint32_t* at)
{
    __shared__ uint32_t place[kSortWaves][1 << kMostBits];
    __shared__ uint32_t sums[kSortWaves];
    const int values = 1 << p.bits, wave = threadIdx.x / kWave, lane = lane_id();
    for (int k = threadIdx.x; k < kSortWaves * values; k += kSortBlock) place[k / values][k % values] = 0;
    __syncthreads();
    const int64_t run = p.tile / kSortWaves, begin = blockIdx.x * p.tile + wave * run;
    for (int64_t k = lane; k < run; k += kWave)
        if (begin + k < p.n) atomicAdd(&place[wave][(key_of(t, begin + k) >> shift) & (values - 1)], 1u);
    __syncthreads();

    // thread v: items with digit v in all tiles, and in the tiles before this one
    uint32_t all = 0, before = 0;
    if ((int)threadIdx.x < values)
        for (int64_t b = 0; b < p.tiles; ++b) {
            const uint32_t k = counts[b * values + threadIdx.x];
            all += k;
            before += b < (int64_t)blockIdx.x ? k : 0;
        }
    // exclusive sum of `all` over the digits
    uint32_t upto = all;
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t k = __shfl_up(upto, d);
        upto += lane >= d ? k : 0;
    }
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    uint32_t base = upto - all + before;
    for (int w = 0; w < wave; ++w) base += sums[w];
    if ((int)threadIdx.x < values)
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t k = place[w][threadIdx.x];
            place[w][threadIdx.x] = base;
            base += k;
        }
    __syncthreads();

    for (int64_t k = 0; k < run && begin + k < p.n; k += kWave) {
        const int64_t i = begin + k + lane;
        const bool here = i < p.n;
        const uint32_t key = here ? key_of(t, i) : 0, digit = (key >> shift) & (values - 1);
        uint64_t same = __ballot(here);
        for (int b = 0; b < p.bits; ++b) {
            const uint64_t ones = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? ones : ~ones;
        }
        const uint64_t lower = same & ((1ull << lane) - 1);
        const uint32_t first = here ? place[wave][digit] : 0;
        wave_sync();
        if (here) {
            const uint32_t to = first + (uint32_t)__popcll(lower);
            keys[to] = key;
            at[to] = t.ids ? (uint32_t)i : t.at[i];
            if (!lower) place[wave][digit] = first + (uint32_t)__popcll(same);
        }
        wave_sync();
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
// the chunk after to partial row 1.
template <class T, class X>
__global__ void __launch_bounds__(kRowBlock) sum_kernel(SumArgs a, const X* dx, T* table)
{
    const int64_t c = ((int64_t)blockIdx.x << (8 - a.gbits)) + (threadIdx.x >> a.gbits);
    const int64_t col = (((int64_t)blockIdx.y << a.gbits) + (threadIdx.x & ((1 << a.gbits) - 1))) * 4;
    if (c >= a.chunks || col >= a.dim) return;
    const int n = a.dim - col < 4 ? (int)(a.dim - col) : 4;
    const int64_t begin = c * a.chunk, end = begin + a.chunk < a.n ? begin + a.chunk : a.n;
    float* part = a.part + c * 2 * a.part_row + col;
    uint32_t key = a.keys[begin];
    bool open = begin > 0 && a.keys[begin - 1] == key;     // the first run began before this chunk
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t i = begin; i < end; ++i) {
        const uint32_t k = a.keys[i];
        if (k != key) {
            if (open)
                store4(part, sum);
            else
                finish_row(a, table, key, col, n, sum);
            open = false;
            key = k;
            sum = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (k >= a.vocab) return;                           // sorted last: no row of the table
        const X* from = dx + (int64_t)a.at[i] * a.x_stride + col;
        sum = sum + widen(n == 4 ? load4(from) : load_some(from, n));
    }
    if (open)
        store4(part, sum);
    else if (end < a.n && a.keys[end] == key)
        store4(part + a.part_row, sum);
    else
        finish_row(a, table, key, col, n, sum);
}

// The runs that cross chunks: the group of the chunk in which one begins adds
// up its partial rows in order.
template <class T>
__global__ void __launch_bounds__(kRowBlock) join_kernel(SumArgs a, T* table)
{
    const int64_t c = ((int64_t)blockIdx.x << (8 - a.gbits)) + (threadIdx.x >> a.gbits);
    const int64_t col = (((int64_t)blockIdx.y << a.gbits) + (threadIdx.x & ((1 << a.gbits) - 1))) * 4;
    if (c >= a.chunks || col >= a.dim) return;
    const int n = a.dim - col < 4 ? (int)(a.dim - col) : 4;
    const int64_t begin = c * a.chunk;
    int64_t end = begin + a.chunk;
    if (end >= a.n) return;
    const uint32_t key = a.keys[end - 1];
    if (key >= a.vocab || a.keys[end] != key) return;                              // ends here
    if (a.keys[begin] == key && begin > 0 && a.keys[begin - 1] == key) return;    // began before
    const float* part = a.part + c * 2 * a.part_row + col;
    v4f sum = load4(part + a.part_row);
    do {
        part += 2 * a.part_row;
        sum = sum + load4(part);
        end += a.chunk;
    } while (end < a.n && a.keys[end] == key);
    finish_row(a, table, key, col, n, sum);
}

template <class T>
__global__ void __launch_bounds__(kRowBlock) zero_rows_kernel(T* table, int64_t vocab, int64_t dim, int64_t stride, int gbits)
{
    const int64_t rows = (int64_t)gridDim.x << (8 - gbits);
    const int lane = threadIdx.x & ((1 << gbits) - 1);
    const typename Quad<T>::vec zero = narrow<T>(v4f{0.0f, 0.0f, 0.0f, 0.0f});
    for (int64_t i = ((int64_t)blockIdx.x << (8 - gbits)) + (threadIdx.x >> gbits); i < vocab; i += rows)
        for (int64_t k = lane * 4; k < dim; k += (int64_t)4 << gbits) {
            if (dim - k >= 4)
                store4(table + i * stride + k, zero);
            else
                store_some(table + i * stride + k, zero, (int)(dim - k));
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

GradPlan grad_plan(const ea_embed_t& c)
{
    GradPlan p{};
    if (c.tokens == 0) return p;
    p.sort = sort_plan(c);
    p.chunk = 32;
    while (c.tokens / p.chunk >= 65536) p.chunk *= 2;
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
    off += align16(p.sort.tiles * ((int64_t)4 << p.sort.bits));
    p.off_part = off;
    off += p.chunks * 2 * p.part_row * 4;
    p.bytes = off;
    return p;
}

// Workgroups for `rows` rows, one group of lanes each; kernels loop over the rest.
unsigned row_groups(int64_t rows, int gbits)
{
    const int64_t per = (int64_t)1 << (8 - gbits), blocks = (rows + per - 1) / per;
    return (unsigned)(blocks < (1 << 22) ? blocks : (1 << 22));
}

template <class T, class X>
hipError_t start_grad(const ea_embed_t& c, const GradPlan& p, const void* ids, const X* dx, T* table, bool accumulate,
                      char* ws, hipStream_t s)
{
    const int gbits = group_bits(c.dim);
    if (!accumulate)
        hipLaunchKernelGGL(zero_rows_kernel<T>, dim3(row_groups(c.vocab, gbits)), dim3(kRowBlock), 0, s, table, c.vocab,
                           c.dim, c.table_stride, gbits);
    if (c.tokens == 0) return hipGetLastError();
    Items t{ids, nullptr, nullptr, c.index_bits, c.vocab, c.padding};
    uint32_t* counts = (uint32_t*)(ws + p.off_counts);
    for (int k = 0; k < p.sort.passes; ++k) {
        uint32_t* keys = (uint32_t*)(ws + p.off_keys[k & 1]);
        uint32_t* at = (uint32_t*)(ws + p.off_at[k & 1]);
        const int shift = k * p.sort.bits;
        hipLaunchKernelGGL(digits_kernel, dim3((unsigned)p.sort.tiles), dim3(kSortBlock), 0, s, t, p.sort, shift, counts);
        hipLaunchKernelGGL(scatter_kernel, dim3((unsigned)p.sort.tiles), dim3(kSortBlock), 0, s, t, p.sort, shift, counts,
                           keys, at);
        t.ids = nullptr;
        t.keys = keys;
        t.at = at;
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
    a.gbits = gbits;
    a.accumulate = accumulate ? 1 : 0;
    const dim3 grid(row_groups(p.chunks, gbits), (unsigned)((c.dim + ((int64_t)4 << gbits) - 1) >> (2 + gbits)));
    hipLaunchKernelGGL((sum_kernel<T, X>), grid, dim3(kRowBlock), 0, s, a, dx, table);
    if (p.chunks > 1) hipLaunchKernelGGL(join_kernel<T>, grid, dim3(kRowBlock), 0, s, a, table);
    return hipGetLastError();
}

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
        hipLaunchKernelGGL((lookup_kernel<T, X>), dim3(row_groups(c.tokens, gbits)), dim3(kRowBlock), 0, s, c,
                           (const T*)table, ids, (X*)x, gbits);
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
