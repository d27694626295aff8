// ea_layer_norm.hip -- layer norm and its gradient.
//
// A row is held in registers by 1, 4 or 16 waves, 16 elements a lane at most,
// so that every array passes memory once; rows of more than 16,384 columns are
// read again for each of their sums.  The gradient of the weights is a sum over
// rows: each workgroup adds its rows' terms in registers and leaves one partial
// row, and a second launch adds those.  Which rows a workgroup takes depends on
// the sizes alone, so every sum has one order.
//
// The squares are summed of differences from the mean, from the same registers:
// nothing cancels.  Bound by bytes: 65,536 x 1,024 bfloat16 44 us, 6.1 TB/s; the
// gradient with a residual's added 106 us, 5.1 TB/s, of which the partial rows'
// sum is 6.  Few rows are bound by launches: 2,048 x 768 binary32 the gradient 12 us,
// 16 x 768 3 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_layer.hpp"

namespace ea {

namespace {

constexpr int kHeldColumns = 16;                       // a lane's, at most
constexpr int kLongBlock = 1024;                       // threads of a row that is not held

// Elements of a vector: 16 bytes of the narrower type, or four where rows are no whole number of those (TAIL).
template <class X, class Y, bool TAIL>
constexpr int vec_of()
{
    return !TAIL && sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
}

template <class X, class Y, bool TAIL>
constexpr int kVec = vec_of<X, Y, TAIL>();

// A vector moved down by some of its elements, zeros behind.
template <int V, class T>
__device__ __forceinline__ Vec<T, V> moved_down(Vec<T, V> v, int by)
{
    const int bits = by * 8 * (int)sizeof(T), rest = bits & 63;
    if constexpr (sizeof(v) == 16) {
        typedef uint64_t Two __attribute__((ext_vector_type(2)));
        const Two w = __builtin_bit_cast(Two, v);
        const uint64_t low = bits < 64 ? w[0] : w[1], high = bits < 64 ? w[1] : 0;
        const Two moved = {(low >> rest) | (rest ? high << (64 - rest) : 0), high >> rest};
        return __builtin_bit_cast(Vec<T, V>, moved);
    } else {
        return __builtin_bit_cast(Vec<T, V>, __builtin_bit_cast(uint64_t, v) >> rest);
    }
}

constexpr int kTail = 1, kTiny = 2;

// The tail of a lane's vector k of K.
template <bool TAIL, int WAVES, int K>
__device__ __forceinline__ constexpr int tail_of(int k)
{
    return !TAIL || k < K - 1 ? 0 : WAVES * K == 1 ? kTiny : kTail;
}

// The row's vector at column `at`, zeros behind its end.  tail: it may cross the end; it is then the row's last whole
// one, moved down, so that a vector is one load and nothing outside the row is read (kTiny: the row may be shorter than
// one).  (Elements one by one for rows of no whole number of vectors: 65,536 x 1,001 bfloat16 135 us and 378 the
// gradient, this way 47 and 106.)
template <int V, class T>
__device__ __forceinline__ Vec<T, V> row_vec(const T* row, int at, int dim, int tail)
{
    Vec<T, V> v = {};
    if (tail == kTiny && dim < V) {
        v = load_part<V>(row + at, dim - at);
    } else if (at < dim) {
        const int from = !tail || at < dim - V ? at : dim - V;
        v = *(const typename VecOf<T, V>::unaligned*)((const char*)row + (uint32_t)from * (uint32_t)sizeof(T));
        if (tail) v = moved_down<V, T>(v, at - from);
    }
    return v;
}

template <int V, class T>
__device__ __forceinline__ void load_row(float* x, const T* row, int at, int dim, int tail)
{
    if constexpr (sizeof(T) * V > 16) {
        load_row<V / 2>(x, row, at, dim, tail);
        load_row<V / 2>(x + V / 2, row, at + V / 2, dim, tail);
    } else {
        widen_to<V, T>(x, row_vec<V>(row, at, dim, tail));
    }
}

template <int V, class T>
__device__ __forceinline__ void store_row(T* row, int at, const float* x, int dim, bool tail)
{
    T* to = (T*)((char*)row + (uint32_t)at * (uint32_t)sizeof(T));
    if (at < dim && (!tail || at + V <= dim))
        store_vec<V>(to, narrow_from<V, T>(x));
    else if (tail && at < dim)
        store_part<V>(to, narrow_from<V, T>(x), dim - at);
}

// weight or bias, or what stands for it where there is none
template <int V>
__device__ __forceinline__ void load_weights(float* x, const void* w, int32_t type, int at, int dim, float none,
                                             int tail)
{
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = none;
    if (!w) return;
    if (type == EA_F32)
        load_row<V>(x, (const float*)w, at, dim, tail);
    else if (type == EA_BF16)
        load_row<V>(x, (const bf16*)w, at, dim, tail);
    else
        load_row<V>(x, (const f16*)w, at, dim, tail);
}

// Floats of a partial row of dweight, and of dbias behind it: whole vectors, what lies behind the columns is not looked
// at.
__host__ __device__ constexpr int64_t partial_row(int64_t dim)
{
    return (dim + 7) / 8 * 8;
}

// Sums of one or two values over the waves of a row; every thread gets them.
template <int WAVES>
__device__ __forceinline__ void row_sums(float& a, float& b, float2* lds)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if (WAVES == 1) return;
    const int wave = wave_id();
    if (lane_id() == 0) lds[wave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
        a = a + lds[k].x;
        b = b + lds[k].y;
    }
    __syncthreads();
}

template <int WAVES>
__device__ __forceinline__ float row_sum(float a, float2* lds)
{
    float none = 0.0f;
    if (WAVES == 1) return wave_sum(a);
    row_sums<WAVES>(a, none, lds);
    return a;
}

// ---- forward --------------------------------------------------------------------

template <class X, class Y, bool TAIL, int WAVES, int K>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave)
    norm_kernel(ea_layer_norm_t c, const X* x, const void* weight, const void* bias, Y* y, float* mean, float* rstd)
{
    constexpr int V = vec_of<X, Y, TAIL>(), kRows = WAVES == 1 ? 4 : 1;          // of a workgroup
    __shared__ float2 lds[WAVES];
    const int lane = WAVES == 1 ? lane_id() : (int)threadIdx.x, dim = (int)c.dim;
    float w[K * V], b[K * V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = (k * WAVES * kWave + lane) * V;
        load_weights<V>(w + k * V, weight, c.w_type, at, dim, 1.0f, tail_of<TAIL, WAVES, K>(k));
        load_weights<V>(b + k * V, bias, c.w_type, at, dim, 0.0f, tail_of<TAIL, WAVES, K>(k));
    }
    const float each = 1.0f / (float)dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave_id() : 0); row < c.rows;
         row += (int64_t)gridDim.x * kRows) {
        float v[K * V], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            load_row<V>(v + k * V, x + row * c.x_stride, (k * WAVES * kWave + lane) * V, dim,
                        tail_of<TAIL, WAVES, K>(k));
#pragma unroll
        for (int k = 0; k < K * V; ++k) sum = sum + v[k];
        const float mu = row_sum<WAVES>(sum, lds) * each;
        float squares = 0.0f;
#pragma unroll
        for (int k = 0; k < K * V; ++k) {
            v[k] = v[k] - mu;
            if (((k / V) * WAVES * kWave + lane) * V + (TAIL && k / V == K - 1 ? k % V : 0) < dim)
                squares = __builtin_fmaf(v[k], v[k], squares);
        }
        const float r = 1.0f / sqrtf(row_sum<WAVES>(squares, lds) * each + c.eps);
#pragma unroll
        for (int k = 0; k < K * V; ++k) v[k] = __builtin_fmaf(v[k] * r, w[k], b[k]);
#pragma unroll
        for (int k = 0; k < K; ++k)
            store_row<V>(y + row * c.y_stride, (k * WAVES * kWave + lane) * V, v + k * V, dim,
                         tail_of<TAIL, WAVES, K>(k));
        if (lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

// Rows too long to hold: a workgroup a row, read once for each sum and once more.
template <class X, class Y, bool TAIL>
__global__ void __launch_bounds__(kLongBlock)
    norm_long_kernel(ea_layer_norm_t c, const X* x, const void* weight, const void* bias, Y* y, float* mean,
                     float* rstd)
{
    constexpr int V = vec_of<X, Y, TAIL>();
    __shared__ float2 lds[kLongBlock / kWave];
    const int dim = (int)c.dim;
    const float each = 1.0f / (float)dim;
    for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
        const X* from = x + row * c.x_stride;
        Y* to = y + row * c.y_stride;
        float v[V], sum = 0.0f, squares = 0.0f;
        for (int at = threadIdx.x * V; at < dim; at += kLongBlock * V) {
            load_row<V>(v, from, at, dim, TAIL ? kTail : 0);
#pragma unroll
            for (int k = 0; k < V; ++k) sum = sum + v[k];
        }
        const float mu = row_sum<kLongBlock / kWave>(sum, lds) * each;
        for (int at = threadIdx.x * V; at < dim; at += kLongBlock * V) {
            load_row<V>(v, from, at, dim, TAIL ? kTail : 0);
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (!TAIL || at + k < dim) squares = __builtin_fmaf(v[k] - mu, v[k] - mu, squares);
        }
        const float r = 1.0f / sqrtf(row_sum<kLongBlock / kWave>(squares, lds) * each + c.eps);
        for (int at = threadIdx.x * V; at < dim; at += kLongBlock * V) {
            float w[V], b[V];
            load_weights<V>(w, weight, c.w_type, at, dim, 1.0f, TAIL ? kTail : 0);
            load_weights<V>(b, bias, c.w_type, at, dim, 0.0f, TAIL ? kTail : 0);
            load_row<V>(v, from, at, dim, TAIL ? kTail : 0);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = __builtin_fmaf((v[k] - mu) * r, w[k], b[k]);
            store_row<V>(to, at, v, dim, TAIL ? kTail : 0);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

// ---- gradient ---------------------------------------------------------------------

// Whether the next row's vectors are asked for before this row's sums are formed.  The registers for them pay where a
// lane holds few columns (131,072 x 256 bfloat16 65 us without, 55 with) and for rows with a tail, whose loads are more
// and smaller (65,536 x 1,001 119 without, 106 with); not for 16 whole columns a lane (32,768 x 1,024 float32 104
// without, 112 with; 65,536 x 1,024 bfloat16 107 either way), nor for 16 waves, which have 128 registers each (4,096 x
// 16,384 149 without, 196 with).
constexpr bool grad_ahead(int waves, int columns, bool tail)
{
    return waves <= 4 && (columns <= 8 || tail);
}

// Waves of a SIMD that the gradient's registers leave room for (four and spills for 1,001 columns: 230 us).
constexpr int grad_waves(int waves, int columns, bool tail)
{
    return grad_ahead(waves, columns, tail) && columns > 8 ? 3 : 4;
}

template <class X, class Y, bool TAIL, int WAVES, int K>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave, (grad_waves(WAVES, K * kVec<X, Y, TAIL>, TAIL)))
    norm_grad_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const void* weight, const float* mean,
                     const float* rstd, const X* add, X* dx, float* partial)
{
    constexpr int V = vec_of<X, Y, TAIL>(), kRows = WAVES == 1 ? 4 : 1;
    // The weights wait in LDS then.
    constexpr bool kAhead = grad_ahead(WAVES, K * V, TAIL);
    __shared__ float2 lds[WAVES];
    __shared__ float weights[kAhead ? WAVES * kWave * K * V : 1];
    const int lane = WAVES == 1 ? lane_id() : (int)threadIdx.x, dim = (int)c.dim;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave_id() : 0);
    Vec<X, V> xr[K];
    Vec<Y, V> yr[K];
    auto load = [&](int64_t from) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * WAVES * kWave + lane) * V, tail = tail_of<TAIL, WAVES, K>(k);
            xr[k] = row_vec<V>(x + from * c.x_stride, at, dim, tail);
            yr[k] = row_vec<V>(dy + from * c.y_stride, at, dim, tail);
        }
    };
    if (kAhead) load(row < c.rows ? row : 0);
    float w[kAhead ? 1 : K * V], dw[K * V], db[K * V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = (k * WAVES * kWave + lane) * V, tail = tail_of<TAIL, WAVES, K>(k);
        if constexpr (kAhead) {
            float some[V];
            load_weights<V>(some, weight, c.w_type, at, dim, 1.0f, tail);
            if (WAVES > 1 || wave_id() == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) weights[at + i] = some[i];
            }
        } else {
            load_weights<V>(w + k * V, weight, c.w_type, at, dim, 1.0f, tail);
        }
    }
    if (kAhead) __syncthreads();
#pragma unroll
    for (int k = 0; k < K * V; ++k) dw[k] = db[k] = 0.0f;
    const float each = 1.0f / (float)dim;
    for (; row < c.rows; row += step) {
        if (!kAhead) load(row);
        const float mu = mean[row], r = rstd[row];
        float v[K * V], d[K * V];
        Vec<X, V> ar[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * WAVES * kWave + lane) * V, tail = tail_of<TAIL, WAVES, K>(k);
            widen_to<V, X>(v + k * V, xr[k]);
            widen_to<V, Y>(d + k * V, yr[k]);
            if (kAhead && add) ar[k] = row_vec<V>(add + row * c.x_stride, at, dim, tail);
        }
        // (the last row's turn asks for that row again)
        if (kAhead) load(row + step < c.rows ? row + step : row);
        float first = 0.0f, second = 0.0f;
#pragma unroll
        for (int k = 0; k < K * V; ++k) {
            v[k] = (v[k] - mu) * r;
            db[k] = db[k] + d[k];
            dw[k] = __builtin_fmaf(d[k], v[k], dw[k]);
            d[k] = d[k] * (kAhead ? weights[(k / V * WAVES * kWave + lane) * V + k % V] : w[kAhead ? 0 : k]);
            first = first + d[k];
            second = __builtin_fmaf(d[k], v[k], second);
        }
        row_sums<WAVES>(first, second, lds);
        first = first * each;
        second = second * each;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * WAVES * kWave + lane) * V, tail = tail_of<TAIL, WAVES, K>(k);
            float o[V];
            if (add) widen_to<V, X>(o, kAhead ? ar[k] : row_vec<V>(add + row * c.x_stride, at, dim, tail));
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float g = (d[k * V + i] - first - v[k * V + i] * second) * r;
                o[i] = add ? o[i] + g : g;
            }
            store_row<V>(dx + row * c.x_stride, at, o, dim, tail);
        }
    }
    if (!partial) return;
    // A workgroup of one-wave rows joins its waves' sums, wave by wave.
    const int64_t held = partial_row(c.dim);
    float* mine = partial + (int64_t)blockIdx.x * 2 * held;
    if constexpr (WAVES == 1) {
        __shared__ float sums[4][2 * K * V][kWave];
        const int wave = wave_id();
#pragma unroll
        for (int k = 0; k < K * V; ++k) {
            sums[wave][k][lane] = dw[k];
            sums[wave][K * V + k][lane] = db[k];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int k = 0; k < K * V; ++k) {
#pragma unroll
            for (int i = 1; i < 4; ++i) {
                dw[k] = dw[k] + sums[i][k][lane];
                db[k] = db[k] + sums[i][K * V + k][lane];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = (k * WAVES * kWave + lane) * V;
        store_row<V>(mine, at, dw + k * V, dim, 0);
        store_row<V>(mine + held, at, db + k * V, dim, 0);
    }
}

template <class X, class Y, bool TAIL>
__global__ void __launch_bounds__(kLongBlock)
    norm_grad_long_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const void* weight, const float* mean,
                          const float* rstd, const X* add, X* dx)
{
    constexpr int V = vec_of<X, Y, TAIL>();
    __shared__ float2 lds[kLongBlock / kWave];
    const int dim = (int)c.dim;
    const float each = 1.0f / (float)dim;
    for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
        const float mu = mean[row], r = rstd[row];
        const X* from = x + row * c.x_stride;
        const Y* grad = dy + row * c.y_stride;
        float v[V], d[V], w[V], first = 0.0f, second = 0.0f;
        for (int at = threadIdx.x * V; at < dim; at += kLongBlock * V) {
            load_weights<V>(w, weight, c.w_type, at, dim, 1.0f, TAIL ? kTail : 0);
            load_row<V>(v, from, at, dim, TAIL ? kTail : 0);
            load_row<V>(d, grad, at, dim, TAIL ? kTail : 0);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                first = first + d[k] * w[k];
                second = __builtin_fmaf(d[k] * w[k], (v[k] - mu) * r, second);
            }
        }
        row_sums<kLongBlock / kWave>(first, second, lds);
        first = first * each;
        second = second * each;
        for (int at = threadIdx.x * V; at < dim; at += kLongBlock * V) {
            float o[V];
            load_weights<V>(w, weight, c.w_type, at, dim, 1.0f, TAIL ? kTail : 0);
            load_row<V>(v, from, at, dim, TAIL ? kTail : 0);
            load_row<V>(d, grad, at, dim, TAIL ? kTail : 0);
            if (add) load_row<V>(o, add + row * c.x_stride, at, dim, TAIL ? kTail : 0);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float g = (d[k] * w[k] - first - (v[k] - mu) * r * second) * r;
                o[k] = add ? o[k] + g : g;
            }
            store_row<V>(dx + row * c.x_stride, at, o, dim, TAIL ? kTail : 0);
        }
    }
}

// The weights' terms of long rows: a workgroup's columns over a run of rows.
constexpr int kColumnBlock = 256;

template <class X, class Y, bool TAIL>
__global__ void __launch_bounds__(kColumnBlock)
    norm_columns_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const float* mean, const float* rstd,
                        float* partial, int64_t run)
{
    constexpr int V = vec_of<X, Y, TAIL>();
    const int at = (int)(blockIdx.x * kColumnBlock + threadIdx.x) * V, dim = (int)c.dim;
    if (at >= dim) return;
    float dw[V] = {}, db[V] = {}, v[V], d[V];
    const int64_t end = (blockIdx.y + 1) * run < c.rows ? (blockIdx.y + 1) * run : c.rows;
    for (int64_t row = blockIdx.y * run; row < end; ++row) {
        const float mu = mean[row], r = rstd[row];
        load_row<V>(v, x + row * c.x_stride, at, dim, TAIL ? kTail : 0);
        load_row<V>(d, dy + row * c.y_stride, at, dim, TAIL ? kTail : 0);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            db[k] = db[k] + d[k];
            dw[k] = __builtin_fmaf(d[k], (v[k] - mu) * r, dw[k]);
        }
    }
    const int64_t held = partial_row(c.dim);
    float* mine = partial + (int64_t)blockIdx.y * 2 * held;
    store_row<V>(mine, at, dw, dim, 0);
    store_row<V>(mine + held, at, db, dim, 0);
}

// The partial rows' sums: 16 columns of dweight and dbias, taken as one row, a workgroup.
constexpr int kJoinColumns = 16, kJoinRows = 64;

__global__ void __launch_bounds__(kJoinColumns* kJoinRows)
    norm_join_kernel(const float* partial, int64_t parts, int64_t dim, void* dweight, void* dbias, int32_t type,
                     int accumulate)
{
    __shared__ float lds[kJoinRows][kJoinColumns + 1];
    const int col = threadIdx.x % kJoinColumns, lane = threadIdx.x / kJoinColumns;
    const int64_t at = (int64_t)blockIdx.x * kJoinColumns + col;
    float sum = 0.0f;
    const int64_t held = partial_row(dim), i = at < dim ? at : at - dim;
    if (at < 2 * dim) {
        const float* from = partial + (at < dim ? 0 : held) + i;
#pragma unroll 4
        for (int64_t k = lane; k < parts; k += kJoinRows) sum = sum + from[k * 2 * held];
    }
    lds[lane][col] = sum;
    __syncthreads();
    for (int half = kJoinRows / 2; half > 0; half /= 2) {
        if (lane < half) lds[lane][col] = lds[lane][col] + lds[lane + half][col];
        __syncthreads();
    }
    if (lane > 0 || at >= 2 * dim) return;
    void* to = at < dim ? dweight : dbias;
    if (!to) return;
    sum = lds[0][col];
    set_element_at(to, type, i, accumulate ? element_at(to, type, i) + sum : sum);
}

// ---- launches -----------------------------------------------------------------------

// Waves of a row and vectors a lane holds of it (0 waves: the row is not held), the fewest that hold it, so that only a
// lane's last vector may cross the row's end; whether one does.
struct Shape {
    int waves, k;
    bool tail;
};

Shape shape_of(const ea_layer_norm_t& c)
{
    const int whole = c.x_type != EA_F32 && c.y_type != EA_F32 ? 8 : 4;
    const bool tail = c.dim % whole != 0;
    const int v = tail ? 4 : whole;
    for (int waves = 1; waves <= 16; waves *= 4)
        for (int k = 1; k * v <= kHeldColumns; ++k)
            if (c.dim <= (int64_t)waves * kWave * k * v) return {waves, k, tail};
    return {0, 0, tail};
}

// f with the tail, the waves and the vectors a lane as constants.
template <int V, class F>
hipError_t with_shape(Shape s, F&& f)
{
#define EA_SHAPE(T, W, K)                           \
    if (s.tail == T && s.waves == W && s.k == K)    \
    return f(std::integral_constant<bool, T>{}, std::integral_constant<int, W>{}, std::integral_constant<int, K>{})
#define EA_WAVES(T, K)   \
    EA_SHAPE(T, 1, K);   \
    EA_SHAPE(T, 4, K);   \
    EA_SHAPE(T, 16, K)
    EA_WAVES(false, 1);
    EA_WAVES(false, 2);
    if constexpr (V == 4) {
        EA_WAVES(false, 3);
        EA_WAVES(false, 4);
    }
    EA_WAVES(true, 1);
    EA_WAVES(true, 2);
    EA_WAVES(true, 3);
    EA_WAVES(true, 4);
#undef EA_WAVES
#undef EA_SHAPE
    return hipErrorInvalidValue;
}

int64_t at_most(int64_t n, int64_t most)
{
    return n < most ? n : most;
}

// Workgroups of the forward pass and of the gradient.
int64_t norm_groups_of(const ea_layer_norm_t& c, Shape s)
{
    return s.waves == 1 ? at_most((c.rows + 3) / 4, 2048) : at_most(c.rows, s.waves == 4 ? 2048 : 512);
}

int64_t grad_groups_of(const ea_layer_norm_t& c, Shape s)
{
    const int columns = s.k * (s.tail || c.x_type == EA_F32 || c.y_type == EA_F32 ? 4 : 8);
    const int64_t held = s.waves == 16 ? 256 : 256 * grad_waves(s.waves, columns, s.tail);
    return at_most(s.waves == 1 ? (c.rows + 3) / 4 : c.rows, held);
}

// Runs of rows of long rows' column sums.
int64_t runs_of(const ea_layer_norm_t& c)
{
    return at_most((c.rows + 15) / 16, 64);
}

}  // namespace

int64_t layer_norm_workspace_bytes(const ea_layer_norm_t& c)
{
    const Shape s = shape_of(c);
    return (s.waves ? grad_groups_of(c, s) : runs_of(c)) * 2 * partial_row(c.dim) * 4;
}

hipError_t launch_layer_norm(const ea_layer_norm_t& c, const void* x, const void* weight, const void* bias, void* y,
                             float* mean, float* rstd, hipStream_t s)
{
    if (c.rows == 0) return hipSuccess;
    const Shape shape = shape_of(c);
    return with_type(c.x_type, [&](auto xt) {
        return with_type(c.y_type, [&](auto yt) {
            using X = decltype(xt);
            using Y = decltype(yt);
            if (!shape.waves) {
                auto* kernel = shape.tail ? norm_long_kernel<X, Y, true> : norm_long_kernel<X, Y, false>;
                hipLaunchKernelGGL(kernel, dim3((unsigned)at_most(c.rows, 1024)), dim3(kLongBlock), 0, s, c,
                                   (const X*)x, weight, bias, (Y*)y, mean, rstd);
                return hipGetLastError();
            }
            const unsigned groups = (unsigned)norm_groups_of(c, shape);
            return with_shape<vec_of<X, Y, false>()>(shape, [&](auto t, auto w, auto k) {
                constexpr int W = decltype(w)::value, K = decltype(k)::value;
                constexpr bool T = decltype(t)::value;
                hipLaunchKernelGGL((norm_kernel<X, Y, T, W, K>), dim3(groups), dim3(W == 1 ? 256 : W * kWave), 0, s, c,
                                   (const X*)x, weight, bias, (Y*)y, mean, rstd);
                return hipGetLastError();
            });
        });
    });
}

hipError_t launch_layer_norm_grad(const ea_layer_norm_t& c, const void* x, const void* dy, const void* weight,
                                  const float* mean, const float* rstd, const void* add, void* dx, void* dweight,
                                  void* dbias, bool accumulate, void* workspace, hipStream_t s)
{
    float* partial = dweight || dbias ? (float*)workspace : nullptr;
    const Shape shape = shape_of(c);
    const int64_t parts = c.rows == 0 ? 0 : shape.waves ? grad_groups_of(c, shape) : runs_of(c);
    hipError_t e = hipSuccess;
    if (c.rows > 0)
        e = with_type(c.x_type, [&](auto xt) {
            return with_type(c.y_type, [&](auto yt) {
                using X = decltype(xt);
                using Y = decltype(yt);
                if (!shape.waves) {
                    const int64_t run = (c.rows + parts - 1) / parts;
                    const int64_t strip = kColumnBlock * (shape.tail ? 4 : vec_of<X, Y, false>());
                    auto* columns = shape.tail ? norm_columns_kernel<X, Y, true> : norm_columns_kernel<X, Y, false>;
                    auto* rows = shape.tail ? norm_grad_long_kernel<X, Y, true> : norm_grad_long_kernel<X, Y, false>;
                    // first: dx may take dy's place
                    if (partial)
                        hipLaunchKernelGGL(columns, dim3((unsigned)((c.dim + strip - 1) / strip), (unsigned)parts),
                                           dim3(kColumnBlock), 0, s, c, (const X*)x, (const Y*)dy, mean, rstd, partial,
                                           run);
                    hipLaunchKernelGGL(rows, dim3((unsigned)at_most(c.rows, 1024)), dim3(kLongBlock), 0, s, c,
                                       (const X*)x, (const Y*)dy, weight, mean, rstd, (const X*)add, (X*)dx);
                    return hipGetLastError();
                }
                return with_shape<vec_of<X, Y, false>()>(shape, [&](auto t, auto w, auto k) {
                    constexpr int W = decltype(w)::value, K = decltype(k)::value;
                    constexpr bool T = decltype(t)::value;
                    hipLaunchKernelGGL((norm_grad_kernel<X, Y, T, W, K>), dim3((unsigned)parts),
                                       dim3(W == 1 ? 256 : W * kWave), 0, s, c, (const X*)x, (const Y*)dy, weight, mean,
                                       rstd, (const X*)add, (X*)dx, partial);
                    return hipGetLastError();
                });
            });
        });
    if (e != hipSuccess || (!dweight && !dbias)) return e;
    const unsigned groups = (unsigned)((2 * c.dim + kJoinColumns - 1) / kJoinColumns);
    hipLaunchKernelGGL(norm_join_kernel, dim3(groups), dim3(kJoinColumns * kJoinRows), 0, s, partial, parts, c.dim,
                       dweight, dbias, c.w_type, accumulate ? 1 : 0);
    return hipGetLastError();
}

}  // namespace ea
