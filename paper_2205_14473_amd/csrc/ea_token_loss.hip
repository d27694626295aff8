// ea_token_loss.hip -- cross-entropy of tokens and its gradient in one pass over
// the logits.
//
// A row is held in registers, as it is stored, by 1, 4, 8 or 16 waves: its largest
// logit and the sum of exponentials are reductions, and the gradient leaves the
// same registers.  Longer rows are cut into pieces and read twice.  The mean's
// gradient needs the number of tokens that count first: a workgroup counts few
// targets itself, many are counted by a launch of their own.
//
// Bound by bytes: the logits once, their gradient once.  8,192 rows of 50,257
// bfloat16 logits with the gradient: 317 us, 5.2 TB/s (1,131 when the exponentials
// of a pass were kept for the next, which spilled; 458 when each pass makes its
// own).  2,048 rows of 32,000 binary32: 106 us, 5.0 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_layer.hpp"

namespace ea {

namespace {

constexpr float kLog2e = 0x1.715476p+0f;
constexpr int kCountBlock = 1024;
constexpr int64_t kMostCounts = 256;                   // workgroups that count
constexpr int64_t kOwnCount = 16;                      // targets a thread up to which each workgroup counts all itself
constexpr int64_t kMostWaves = 4096;                   // of the main pass, 16 a CU; twice as many where a row is one wave's
constexpr int kEndBlock = 256;

// Workspace: the counting groups' counts, then each main group's sum and count (for rows in pieces each row's, then
// each piece's largest logit and sum, then each row's target's logit).
struct Sums {
    double loss;
    int64_t count;
};
static_assert(sizeof(Sums) == 16, "the workspace's layout");

struct Loss {
    ea_token_loss_t c;
    const void* targets;
    float* loss;
    int64_t* counts;                                   // of `parts` groups, or NULL: the targets are few
    Sums* sums;
    int32_t parts;
    int32_t pieces;                                    // of a row
    float2* ends;                                      // each piece's largest logit and sum
    float* hits;                                       // each row's target's logit
};

// The target of a row, -1 where it does not count.
__device__ __forceinline__ int target_at(const Loss& a, int64_t row)
{
    const int64_t t =
        a.c.index_bits == 64 ? ((const int64_t*)a.targets)[row] : (int64_t)((const int32_t*)a.targets)[row];
    return t >= 0 && t < a.c.vocab ? (int)t : -1;
}

// The workgroup's sum of integers; every thread gets it.
template <int THREADS>
__device__ __forceinline__ int64_t group_count(int64_t v)
{
    __shared__ int64_t lds[THREADS / kWave];
    for (int k = kWave / 2; k > 0; k /= 2) v += __shfl_xor(v, k);
    if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0;
    for (int k = 0; k < THREADS / kWave; ++k) v += lds[k];
    __syncthreads();
    return v;
}

__global__ void __launch_bounds__(kCountBlock) count_kernel(Loss a)
{
    int64_t n = 0;
    for (int64_t i = (int64_t)blockIdx.x * kCountBlock + threadIdx.x; i < a.c.rows;
         i += (int64_t)gridDim.x * kCountBlock)
        n += target_at(a, i) >= 0;
    n = group_count<kCountBlock>(n);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// What the gradient of a row that counts is multiplied by.
template <int THREADS>
__device__ __forceinline__ float row_factor(const Loss& a)
{
    if (a.c.reduction == EA_REDUCE_SUM) return a.c.scale;
    int64_t n = 0;
    if (a.counts) {
        for (int i = threadIdx.x; i < a.parts; i += THREADS) n += a.counts[i];
    } else {
#pragma unroll
        for (int k = 0; k < kOwnCount; ++k) {
            const int64_t i = (int64_t)k * THREADS + threadIdx.x;
            if (i < a.c.rows) n += target_at(a, i) >= 0;
        }
    }
    n = group_count<THREADS>(n);
    return n > 0 ? (float)((double)a.c.scale / (double)n) : 0.0f;
}

template <int WAVES>
__device__ __forceinline__ float group_max(float v, float* lds)
{
    v = wave_max(v);
    if (WAVES == 1) return v;
    if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) v = fmaxf(v, lds[k]);
    return v;
}

template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float* lds)
{
    v = wave_sum(v);
    if (WAVES == 1) return v;
    if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) v = v + lds[k];
    return v;
}

// e^(z - top): the difference is rounded before it is scaled, so that logits near the largest, and large ones, lose
// nothing.
__device__ __forceinline__ float exp_under(float z, float top)
{
    return __builtin_amdgcn_exp2f((z - top) * kLog2e);
}

// Four words of a row made opaque: what a pass made of them (as floats, and their exponentials) is made anew by the
// next one.  Kept, it would take two to four times the registers of the row itself.
typedef uint32_t Words __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void renew(Words& w)
{
    asm volatile("" : "+v"(w));
}

template <class T>
__device__ __forceinline__ void as_floats(float* x, Words w)
{
    constexpr int V = 16 / sizeof(T);
    widen_to<V, T>(x, __builtin_bit_cast(Vec<T, V>, w));
}

// A row as a wave sees it: vectors of 16 bytes on a grid of cache lines, the first of which may begin before the row
// and the last end behind it.  (8,192 rows of 50,257 logits of 16 bits, with the gradient, before the next row was
// asked for early: 442 us with vectors from the row's own start on, 404 with the 16-byte grid, 358 with this one.)
// Bytes of the grid's cells: short rows, one wave each, take a vector's, which costs them fewer vectors.
constexpr int cell_of(int waves)
{
    return waves == 1 ? 16 : 128;
}

template <class T>
struct Grid {
    T* row;                                            // the cell that holds the row's start
    int head, end;                                     // the row's elements from there on: [head, end)
    // the same cells of another row
    template <class O>
    __device__ Grid(T* p, const Grid<O>& like) : row(p - like.head), head(like.head), end(like.end)
    {
    }
    __device__ Grid(T* p, int vocab, int cell)
    {
        head = (int)((uintptr_t)p % (uintptr_t)cell / sizeof(T));
        row = p - head;
        end = vocab + head;
    }
};

// The wave's 64 vectors from element `at` on: all inside, none, or some of their elements.  The piece's address is a
// scalar, kept one for each piece (opaque), and the lane's part of it the same for all: otherwise every piece's address
// takes two registers, which are a third of those that hold the row.
template <class T>
__device__ __forceinline__ T* piece(T* row, int at)
{
    T* p = row + at;
    asm volatile("" : "+s"(p));
    return p;
}

// The wave's vectors, -infinity outside the row.  One that holds an element of the row is read whole: it lies in one
// cell of 16 bytes, and so in memory that is allocated if the element is, and what it holds of others has no effect.
template <class T>
__device__ __forceinline__ Words load_words(const Grid<const T>& g, int at)
{
    constexpr int V = 16 / sizeof(T);
    const T* p = piece(g.row, at);
    const uint32_t off = (uint32_t)lane_id() * 16u;
    if (at >= g.head && at + kWave * V <= g.end) return *(const Words*)((const char*)p + off);
    const int mine = at + lane_id() * V;
    Words w = {};
    if (mine + V > g.head && mine < g.end) w = *(const Words*)((const char*)p + off);
    Vec<T, V> v = __builtin_bit_cast(Vec<T, V>, w);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = mine + k >= g.head && mine + k < g.end ? v[k] : (T)-__builtin_inff();
    return __builtin_bit_cast(Words, v);
}

template <bool ONCE, class T>
__device__ __forceinline__ void store_floats_of(const Grid<T>& g, int at, const float* x)
{
    constexpr int V = 16 / sizeof(T);
    T* p = piece(g.row, at);
    const Vec<T, V> v = narrow_from<V, T>(x);
    const uint32_t off = (uint32_t)lane_id() * 16u;
    if (at >= g.head && at + kWave * V <= g.end) {
        store_vec<V, ONCE>((T*)((char*)p + off), v);
        return;
    }
    const int mine = at + lane_id() * V;
    if (mine >= g.head && mine + V <= g.end) {
        store_vec<V, ONCE>((T*)((char*)p + off), v);
    } else {
        T* q = (T*)((char*)p + off);
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (mine + k >= g.head && mine + k < g.end) q[k] = v[k];
    }
}

template <bool ONCE, class T>
__device__ __forceinline__ void zero_row(const Grid<T>& g, int first, int lanes)
{
    constexpr int V = 16 / sizeof(T);
    const float none[V] = {};
    for (int at = first; at < g.end; at += lanes * V) store_floats_of<ONCE>(g, at, none);
}

// WAVES of a row (1: four rows a workgroup), K vectors of 16 bytes a lane.
// ONCE: the gradient goes past the caches.
template <class T, int WAVES, int K, bool GRAD, bool ONCE>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave, 4)
    loss_kernel(Loss a, const T* logits, T* dlogits)
{
    constexpr int V = 16 / sizeof(T), kRows = WAVES == 1 ? 4 : 1, kLanes = WAVES * kWave;
    constexpr int kThreads = WAVES == 1 ? 256 : kLanes;
    __shared__ float lds[2][WAVES], hit_of[kRows];
    const int lane = WAVES == 1 ? lane_id() : (int)threadIdx.x;
    const int slot = WAVES == 1 ? wave_id() : 0, first = WAVES == 1 ? 0 : wave_id() * kWave * V;
    const int vocab = (int)a.c.vocab;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + slot;
    int target = uniform(row < a.c.rows ? target_at(a, row) : -1);
    const T* from = logits + (row < a.c.rows ? row : 0) * a.c.logits_stride;
    Words z[K];
    auto load = [&](const T* p) {
        const Grid<const T> g(p, vocab, cell_of(WAVES));
#pragma unroll
        for (int k = 0; k < K; ++k) z[k] = load_words(g, k * kLanes * V + first);
    };
    load(from);
    const float factor = GRAD ? row_factor<kThreads>(a) : 0.0f;
    double total = 0.0;
    int64_t used = 0;
    while (row < a.c.rows) {
        // The next row's vectors follow this one's into the same registers as they are used for the last time (where
        // none follows, or one that does not count, this one's again, from the cache): 358 -> 323 us for 8,192 rows.
        const int64_t row_after = row + step;
        const int target_after = uniform(row_after < a.c.rows ? target_at(a, row_after) : -1);
        const T* after = target_after >= 0 ? logits + row_after * a.c.logits_stride : from;
        T* to = dlogits + row * a.c.dlogits_stride;
        if (target < 0) {
            if (lane == 0 && a.loss) a.loss[row] = 0.0f;
            if (GRAD) zero_row<ONCE>(Grid<T>(to, vocab, cell_of(WAVES)), first, kLanes);
            load(after);
        } else {
            const Grid<const T> in(from, vocab, cell_of(WAVES)), next(after, vocab, cell_of(WAVES));
            float top = -__builtin_inff(), sum = 0.0f, x[V];
            // f(vector, the wave's first element of it on the grid) for each of the lane's vectors
            auto every = [&](auto&& f, bool last) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int at = k * kLanes * V + first;
                    renew(z[k]);
                    if (at < in.end) f(z[k], at);
                    if (last) z[k] = load_words(next, at);
                }
            };
            // The target's logit, from one lane before the last reduction: when rows are written where they were read,
            // no lane may still want it after that.
            if (lane == 0) hit_of[slot] = (float)from[target];
            if (WAVES == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (more waves: the reductions')
            every(
                [&](Words w, int) {
                    as_floats<T>(x, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) top = fmaxf(top, x[i]);
                },
                false);
            top = group_max<WAVES>(top, lds[0]);
            every(
                [&](Words w, int) {
                    as_floats<T>(x, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) sum = sum + exp_under(x[i], top);
                },
                !GRAD);
            sum = group_sum<WAVES>(sum, lds[1]);
            const float hit = hit_of[slot], loss = logf(sum) - (hit - top);
            total = total + (double)loss;
            ++used;
            if (lane == 0 && a.loss) a.loss[row] = loss;
            if constexpr (GRAD) {
                const float share = factor / sum;
                // the gradient's rows on the same grid as the logits, whether it is theirs or not
                const Grid<T> out(to, in);
                every(
                    [&](Words w, int at) {
                        as_floats<T>(x, w);
#pragma unroll
                        for (int i = 0; i < V; ++i) x[i] = exp_under(x[i], top) * share;
                        store_floats_of<ONCE>(out, at, x);
                    },
                    true);
                // the lane that wrote the target's element writes it again, less the factor
                if ((target + in.head) / V % kLanes == lane) to[target] = (T)(exp_under(hit, top) * share - factor);
            }
            if (WAVES > 1) __syncthreads();            // the next row's reductions write where this one's were read
        }
        row = row_after;
        target = target_after;
        from = after;
    }
    // one sum for each row's group of waves
    if (lane == 0) a.sums[(int64_t)blockIdx.x * kRows + slot] = Sums{total, used};
}

// Rows too long for registers, in pieces of a workgroup each: the largest logit of a piece and its sum under that,
// then, from those of all pieces, in one order, the loss and the piece's gradient.  (A workgroup a row that reads it again,
// eight vectors ahead, against pieces: 1 row of 250,000 binary32 logits 45 us and 14; 60 of 200,001 47 and 26; 1,000 of
// 100,000 221 and 206.)
constexpr int kPieceWaves = 4, kPieceVectors = 8, kPieceThreads = kPieceWaves * kWave;

template <class T>
constexpr int kPiece = kPieceThreads * kPieceVectors * 16 / (int)sizeof(T);      // elements

template <class T>
__global__ void __launch_bounds__(kPieceThreads) loss_ends_kernel(Loss a, const T* logits)
{
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[2][kPieceWaves];
    const int64_t items = a.c.rows * a.pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = item / a.pieces;
        const int target = uniform(target_at(a, row));
        if (target < 0) continue;
        const T* from = logits + row * a.c.logits_stride;
        const Grid<const T> g(from, (int)a.c.vocab, cell_of(kPieceWaves));
        const int start = (int)(item - row * a.pieces) * kPiece<T>, first = start + wave_id() * kWave * V;
        Words z[kPieceVectors];
#pragma unroll
        for (int k = 0; k < kPieceVectors; ++k) z[k] = load_words(g, first + k * kPieceThreads * V);
        float x[V], top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kPieceVectors; ++k) {
            as_floats<T>(x, z[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) top = fmaxf(top, x[i]);
        }
        top = group_max<kPieceWaves>(top, lds[0]);
        const float base = top == -__builtin_inff() ? 0.0f : top;      // nothing but -infinity: a sum of 0 (NaN: NaN)
#pragma unroll
        for (int k = 0; k < kPieceVectors; ++k) {
            renew(z[k]);
            as_floats<T>(x, z[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) sum = sum + exp_under(x[i], base);
        }
        sum = group_sum<kPieceWaves>(sum, lds[1]);
        if (threadIdx.x == 0) {
            a.ends[item] = make_float2(top, sum);
            const int at = target + g.head - start;
            if (at >= 0 && at < kPiece<T>) a.hits[row] = (float)from[target];
        }
        __syncthreads();                               // the next piece's reductions write where this one's were read
    }
}

template <class T, bool GRAD, bool ONCE>
__global__ void __launch_bounds__(kPieceThreads) loss_pieces_kernel(Loss a, const T* logits, T* dlogits)
{
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[2][kPieceWaves];
    const int64_t items = GRAD ? a.c.rows * a.pieces : a.c.rows;
    const float factor = GRAD ? row_factor<kPieceThreads>(a) : 0.0f;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = GRAD ? item / a.pieces : item;
        const int piece = GRAD ? (int)(item - row * a.pieces) : 0;
        const int target = uniform(target_at(a, row)), vocab = (int)a.c.vocab;
        const T* from = logits + row * a.c.logits_stride;
        const Grid<const T> in(from, vocab, cell_of(kPieceWaves));
        T* to = dlogits + row * a.c.dlogits_stride;
        const Grid<T> out(to, in);
        const int start = piece * kPiece<T>, first = start + wave_id() * kWave * V;
        if (target < 0) {
            if (piece == 0 && threadIdx.x == 0) {
                if (a.loss) a.loss[row] = 0.0f;
                a.sums[row] = Sums{0.0, 0};
            }
            if (GRAD) {
                const float none[V] = {};
#pragma unroll
                for (int k = 0; k < kPieceVectors; ++k) store_floats_of<ONCE>(out, first + k * kPieceThreads * V, none);
            }
            continue;
        }
        Words z[kPieceVectors];
        if (GRAD) {
#pragma unroll
            for (int k = 0; k < kPieceVectors; ++k) z[k] = load_words(in, first + k * kPieceThreads * V);
        }
        const float2* ends = a.ends + row * a.pieces;
        float top = -__builtin_inff(), sum = 0.0f;
        for (int i = threadIdx.x; i < a.pieces; i += kPieceThreads) top = fmaxf(top, ends[i].x);
        top = group_max<kPieceWaves>(top, lds[0]);
        for (int i = threadIdx.x; i < a.pieces; i += kPieceThreads) sum = sum + ends[i].y * exp_under(ends[i].x, top);
        sum = group_sum<kPieceWaves>(sum, lds[1]);
        const float hit = a.hits[row];
        if (piece == 0 && threadIdx.x == 0) {
            const float loss = logf(sum) - (hit - top);
            if (a.loss) a.loss[row] = loss;
            a.sums[row] = Sums{(double)loss, 1};
        }
        if constexpr (GRAD) {
            const float share = factor / sum;
            float x[V];
#pragma unroll
            for (int k = 0; k < kPieceVectors; ++k) {
                as_floats<T>(x, z[k]);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = exp_under(x[i], top) * share;
                store_floats_of<ONCE>(out, first + k * kPieceThreads * V, x);
            }
            // the lane that wrote the target's element writes it again, less the factor
            const int at = target + in.head - start;
            if (at >= 0 && at < kPiece<T> && at / V % kPieceThreads == (int)threadIdx.x)
                to[target] = (T)(exp_under(hit, top) * share - factor);
        }
        __syncthreads();                               // the next piece's reductions write where this one's were read
    }
}

// The groups' sums, in their order.
__global__ void __launch_bounds__(kEndBlock) loss_end_kernel(Loss a, int64_t groups, float* total, int32_t* count)
{
    __shared__ double sums[kEndBlock];
    double sum = 0.0;
    int64_t used = 0;
    for (int64_t i = threadIdx.x; i < groups; i += kEndBlock) {
        sum = sum + a.sums[i].loss;
        used += a.sums[i].count;
    }
    used = group_count<kEndBlock>(used);
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int half = kEndBlock / 2; half > 0; half /= 2) {
        if ((int)threadIdx.x < half) sums[threadIdx.x] = sums[threadIdx.x] + sums[threadIdx.x + half];
        __syncthreads();
    }
    if (threadIdx.x > 0) return;
    sum = sums[0];
    if (a.c.reduction == EA_REDUCE_MEAN && used > 0) sum = sum / (double)used;
    *total = (float)sum;
    if (count) *count = (int32_t)used;
}

int64_t at_most(int64_t n, int64_t most)
{
    return n < most ? n : most;
}

// Waves of a row and vectors a lane: the first that holds it, or those of a piece and 0 where none does.  Few waves with
// many vectors each: rows of their own work beside each other on a CU, one reading or writing while another reduces.
// (From 10 vectors a lane on in steps of two: 13 between 12 and 14 gained 1% at most with the gradient, 2% without.)
// Without the gradient, many forms of 10 vectors and more keep one or two registers in scratch.
struct Shape {
    int waves, k;
};

#define EA_SHAPES                                                                                                  \
    EA_SHAPE(1, 2)                                                                                                 \
    EA_SHAPE(1, 4)                                                                                                 \
    EA_SHAPE(1, 8)                                                                                                 \
    EA_SHAPE(4, 4)                                                                                                 \
    EA_SHAPE(4, 6)                                                                                                 \
    EA_SHAPE(4, 8)                                                                                                 \
    EA_SHAPE(4, 12)                                                                                                \
    EA_SHAPE(4, 16)                                                                                                \
    EA_SHAPE(8, 10)                                                                                                \
    EA_SHAPE(8, 12)                                                                                                \
    EA_SHAPE(8, 14)                                                                                                \
    EA_SHAPE(8, 16)                                                                                                \
    EA_SHAPE(16, 10)                                                                                               \
    EA_SHAPE(16, 12)                                                                                               \
    EA_SHAPE(16, 14)                                                                                               \
    EA_SHAPE(16, 16)

Shape shape_of(const ea_token_loss_t& c)
{
    const int64_t v = c.type == EA_F32 ? 4 : 8;
    const Shape all[] = {
#define EA_SHAPE(W, K) {W, K},
        EA_SHAPES
#undef EA_SHAPE
    };
    for (const Shape& s : all)
        // wherever in a cell a row starts
        if (c.vocab + cell_of(s.waves) / 16 * v - 1 <= v * kWave * s.waves * s.k) return s;
    return {kPieceWaves, 0};
}

// Pieces of a row that is not held, wherever in a cell it starts.
int64_t pieces_of(const ea_token_loss_t& c)
{
    const int64_t size = c.type == EA_F32 ? 4 : 2, piece = kPieceThreads * kPieceVectors * 16 / size;
    return (c.vocab + cell_of(kPieceWaves) / size - 1 + piece - 1) / piece;
}

// Workgroups of the main pass, and the sums they leave.
int64_t groups_of(const ea_token_loss_t& c, Shape s)
{
    return s.waves == 1 ? at_most((c.rows + 3) / 4, kMostWaves / 2) : at_most(c.rows, kMostWaves / s.waves);
}

int64_t sums_of(const ea_token_loss_t& c, Shape s)
{
    return s.k == 0 ? c.rows : groups_of(c, s) * (s.waves == 1 ? 4 : 1);
}

int64_t counting_groups(const ea_token_loss_t& c)
{
    const int waves = shape_of(c).waves, threads = waves == 1 ? 256 : waves * kWave;
    return c.rows > kOwnCount * threads ? at_most((c.rows + kCountBlock * 4 - 1) / (kCountBlock * 4), kMostCounts) : 0;
}

template <class T, bool GRAD, bool ONCE>
hipError_t start_loss(const Loss& a, Shape s, unsigned groups, const void* logits, void* dlogits, hipStream_t st)
{
#define EA_SHAPE(W, K)                                                                                            \
    if (s.waves == W && s.k == K) {                                                                               \
        hipLaunchKernelGGL((loss_kernel<T, W, K, GRAD, ONCE>), dim3(groups), dim3(W == 1 ? 256 : W * kWave), 0,   \
                           st, a, (const T*)logits, (T*)dlogits);                                                 \
        return hipGetLastError();                                                                                 \
    }
    EA_SHAPES
#undef EA_SHAPE
    return hipErrorInvalidValue;
}

template <class T, bool GRAD, bool ONCE>
hipError_t start_pieces(const Loss& a, const void* logits, void* dlogits, hipStream_t st)
{
    const int64_t items = a.c.rows * a.pieces, most = 1 << 20;
    hipLaunchKernelGGL(loss_ends_kernel<T>, dim3((unsigned)at_most(items, most)), dim3(kPieceThreads), 0, st, a,
                       (const T*)logits);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((loss_pieces_kernel<T, GRAD, ONCE>), dim3((unsigned)at_most(GRAD ? items : a.c.rows, most)),
                       dim3(kPieceThreads), 0, st, a, (const T*)logits, (T*)dlogits);
    return hipGetLastError();
}

}  // namespace

int64_t token_loss_workspace_bytes(const ea_token_loss_t& c)
{
    const Shape s = shape_of(c);
    return counting_groups(c) * 16 + sums_of(c, s) * 16 + (s.k == 0 ? c.rows * pieces_of(c) * 8 + c.rows * 4 : 0);
}

hipError_t launch_token_loss(const ea_token_loss_t& c, const void* logits, const void* targets, float* loss,
                             float* total, int32_t* count, void* dlogits, void* workspace, hipStream_t s)
{
    const Shape shape = shape_of(c);
    const int64_t parts = counting_groups(c);
    Loss a{};
    a.c = c;
    a.targets = targets;
    a.loss = loss;
    a.sums = (Sums*)((char*)workspace + parts * 16);
    if (shape.k == 0) {
        a.pieces = (int32_t)pieces_of(c);
        a.ends = (float2*)(a.sums + c.rows);
        a.hits = (float*)(a.ends + c.rows * a.pieces);
    }
    hipError_t e = hipSuccess;
    if (dlogits && c.reduction == EA_REDUCE_MEAN && parts > 0) {
        a.counts = (int64_t*)workspace;
        a.parts = (int32_t)parts;
        hipLaunchKernelGGL(count_kernel, dim3((unsigned)parts), dim3(kCountBlock), 0, s, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && c.rows > 0)
        e = with_type(c.type, [&](auto t) {
            using T = decltype(t);
            const unsigned groups = (unsigned)groups_of(c, shape);
            if (!dlogits)
                return shape.k ? start_loss<T, false, false>(a, shape, groups, logits, dlogits, s)
                               : start_pieces<T, false, false>(a, logits, dlogits, s);
            return with_bool(past_caches(c.rows * c.vocab, c.type), [&](auto once) {
                constexpr bool O = decltype(once)::value;
                return shape.k ? start_loss<T, true, O>(a, shape, groups, logits, dlogits, s)
                               : start_pieces<T, true, O>(a, logits, dlogits, s);
            });
        });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(loss_end_kernel, dim3(1), dim3(kEndBlock), 0, s, a, sums_of(c, shape), total, count);
    return hipGetLastError();
}

}  // namespace ea
