// ea_layer_norm.hip -- layer norm and its gradient.
//
// A row is held in registers by 1, 4 or 16 waves, 16 elements a lane at most,
// so that every array passes memory once; rows of more than 16,384 columns are
// read again for each of their sums.  The gradient of the weights is a sum over
// rows: each workgroup adds its rows' terms in registers and leaves one partial
// row, and a second launch adds those.  Which rows a workgroup takes depends on
// the sizes alone, so every sum has one order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_layer.hpp"

namespace ea {

namespace {

constexpr int kHeldColumns = 16;                       // a lane's, at most
constexpr int kLongBlock = 1024;                       // threads of a row that is not held

template <class X, class Y>
constexpr int vec_of()
{
    return sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
}

// Elements of a vector at column `at` that lie inside the row.
template <int V>
__device__ __forceinline__ int inside(int64_t at, int64_t dim)
{
    const int64_t left = dim - at;
    return left >= V ? V : left > 0 ? (int)left : 0;
}

template <int V, class T>
__device__ __forceinline__ void load_some_of(float* x, const T* row, int64_t at, int n)
{
    if (n == V)
        widen_to<V, T>(x, load_vec<V>(row + at));
    else
        widen_to<V, T>(x, load_part<V>(row + at, n));
}

template <int V, class T>
__device__ __forceinline__ void store_some_of(T* row, int64_t at, const float* x, int n)
{
    if (n == V)
        store_vec<V>(row + at, narrow_from<V, T>(x));
    else
        store_part<V>(row + at, narrow_from<V, T>(x), n);
}

// weight or bias, or what stands for it where there is none
template <int V>
__device__ __forceinline__ void load_weights(float* x, const void* w, int32_t type, int64_t at, int n, float none)
{
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = none;
    if (!w || n == 0) return;
    if (type == EA_F32)
        load_some_of<V>(x, (const float*)w, at, n);
    else if (type == EA_BF16)
        load_some_of<V>(x, (const bf16*)w, at, n);
    else
        load_some_of<V>(x, (const f16*)w, at, n);
}

// Sums of one or two values over the waves of a row; every thread gets them.
template <int WAVES>
__device__ __forceinline__ void row_sums(float& a, float& b, float2* lds)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if (WAVES == 1) return;
    const int wave = threadIdx.x / kWave;
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

template <class X, class Y, int WAVES, int K>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave)
    norm_kernel(ea_layer_norm_t c, const X* x, const void* weight, const void* bias, Y* y, float* mean, float* rstd)
{
    constexpr int V = vec_of<X, Y>();
    constexpr int kRows = WAVES == 1 ? 4 : 1;          // of a workgroup
    __shared__ float2 lds[WAVES];
    const int lane = WAVES == 1 ? lane_id() : (int)threadIdx.x;
    float w[K * V], b[K * V];
    int n[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t at = (int64_t)(k * WAVES * kWave + lane) * V;
        n[k] = inside<V>(at, c.dim);
        load_weights<V>(w + k * V, weight, c.w_type, at, n[k], 1.0f);
        load_weights<V>(b + k * V, bias, c.w_type, at, n[k], 0.0f);
    }
    const float each = 1.0f / (float)c.dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? threadIdx.x / kWave : 0); row < c.rows;
         row += (int64_t)gridDim.x * kRows) {
        float v[K * V], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            load_some_of<V>(v + k * V, x + row * c.x_stride, (int64_t)(k * WAVES * kWave + lane) * V, n[k]);
#pragma unroll
        for (int k = 0; k < K * V; ++k) sum = sum + v[k];
        const float mu = row_sum<WAVES>(sum, lds) * each;
        float squares = 0.0f;
#pragma unroll
        for (int k = 0; k < K * V; ++k) {
            v[k] = v[k] - mu;
            if (k % V < n[k / V]) squares = __builtin_fmaf(v[k], v[k], squares);
        }
        const float r = 1.0f / sqrtf(row_sum<WAVES>(squares, lds) * each + c.eps);
#pragma unroll
        for (int k = 0; k < K * V; ++k) v[k] = __builtin_fmaf(v[k] * r, w[k], b[k]);
#pragma unroll
        for (int k = 0; k < K; ++k)
            store_some_of<V>(y + row * c.y_stride, (int64_t)(k * WAVES * kWave + lane) * V, v + k * V, n[k]);
        if (lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

// Rows too long to hold: a workgroup a row, read once for each sum and once more.
template <class X, class Y>
__global__ void __launch_bounds__(kLongBlock)
    norm_long_kernel(ea_layer_norm_t c, const X* x, const void* weight, const void* bias, Y* y, float* mean, float* rstd)
{
    constexpr int V = vec_of<X, Y>();
    __shared__ float2 lds[kLongBlock / kWave];
    const float each = 1.0f / (float)c.dim;
    for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
        const X* from = x + row * c.x_stride;
        Y* to = y + row * c.y_stride;
        float v[V], sum = 0.0f, squares = 0.0f;
        for (int64_t at = threadIdx.x * V; at < c.dim; at += kLongBlock * V) {
            load_some_of<V>(v, from, at, inside<V>(at, c.dim));
#pragma unroll
            for (int k = 0; k < V; ++k) sum = sum + v[k];
        }
        const float mu = row_sum<kLongBlock / kWave>(sum, lds) * each;
        for (int64_t at = threadIdx.x * V; at < c.dim; at += kLongBlock * V) {
            const int n = inside<V>(at, c.dim);
            load_some_of<V>(v, from, at, n);
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < n) squares = __builtin_fmaf(v[k] - mu, v[k] - mu, squares);
        }
        const float r = 1.0f / sqrtf(row_sum<kLongBlock / kWave>(squares, lds) * each + c.eps);
        for (int64_t at = threadIdx.x * V; at < c.dim; at += kLongBlock * V) {
            const int n = inside<V>(at, c.dim);
            float w[V], b[V];
            load_weights<V>(w, weight, c.w_type, at, n, 1.0f);
            load_weights<V>(b, bias, c.w_type, at, n, 0.0f);
            load_some_of<V>(v, from, at, n);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = __builtin_fmaf((v[k] - mu) * r, w[k], b[k]);
            store_some_of<V>(to, at, v, n);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

// ---- gradient ---------------------------------------------------------------------

template <class X, class Y, int WAVES, int K>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave)
    norm_grad_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const void* weight, const float* mean,
                     const float* rstd, const X* add, X* dx, float* partial)
{
    constexpr int V = vec_of<X, Y>();
    constexpr int kRows = WAVES == 1 ? 4 : 1;
    __shared__ float2 lds[WAVES];
    const int lane = WAVES == 1 ? lane_id() : (int)threadIdx.x;
    float w[K * V], dw[K * V], db[K * V];
    int n[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t at = (int64_t)(k * WAVES * kWave + lane) * V;
        n[k] = inside<V>(at, c.dim);
        load_weights<V>(w + k * V, weight, c.w_type, at, n[k], 1.0f);
    }
#pragma unroll
    for (int k = 0; k < K * V; ++k) dw[k] = db[k] = 0.0f;
    const float each = 1.0f / (float)c.dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? threadIdx.x / kWave : 0); row < c.rows;
         row += (int64_t)gridDim.x * kRows) {
        float v[K * V], d[K * V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t at = (int64_t)(k * WAVES * kWave + lane) * V;
            load_some_of<V>(v + k * V, x + row * c.x_stride, at, n[k]);
            load_some_of<V>(d + k * V, dy + row * c.y_stride, at, n[k]);
        }
        const float mu = mean[row], r = rstd[row];
        float first = 0.0f, second = 0.0f;
#pragma unroll
        for (int k = 0; k < K * V; ++k) {
            v[k] = (v[k] - mu) * r;
            db[k] = db[k] + d[k];
            dw[k] = __builtin_fmaf(d[k], v[k], dw[k]);
            d[k] = d[k] * w[k];
            first = first + d[k];
            second = __builtin_fmaf(d[k], v[k], second);
        }
        row_sums<WAVES>(first, second, lds);
        first = first * each;
        second = second * each;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t at = (int64_t)(k * WAVES * kWave + lane) * V;
            float o[V];
            if (add) load_some_of<V>(o, add + row * c.x_stride, at, n[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float g = (d[k * V + i] - first - v[k * V + i] * second) * r;
                o[i] = add ? o[i] + g : g;
            }
            store_some_of<V>(dx + row * c.x_stride, at, o, n[k]);
        }
    }
    if (!partial) return;
    // A workgroup of one-wave rows joins its waves' sums, wave by wave.
    float* mine = partial + (int64_t)blockIdx.x * 2 * c.dim;
    if constexpr (WAVES == 1) {
        __shared__ float sums[4][2 * K * V][kWave];
        const int wave = threadIdx.x / kWave;
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
        const int64_t at = (int64_t)(k * WAVES * kWave + lane) * V;
        store_some_of<V>(mine, at, dw + k * V, n[k]);
        store_some_of<V>(mine + c.dim, at, db + k * V, n[k]);
    }
}

template <class X, class Y>
__global__ void __launch_bounds__(kLongBlock)
    norm_grad_long_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const void* weight, const float* mean,
                          const float* rstd, const X* add, X* dx)
{
    constexpr int V = vec_of<X, Y>();
    __shared__ float2 lds[kLongBlock / kWave];
    const float each = 1.0f / (float)c.dim;
    for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
        const float mu = mean[row], r = rstd[row];
        const X* from = x + row * c.x_stride;
        const Y* grad = dy + row * c.y_stride;
        float v[V], d[V], w[V], first = 0.0f, second = 0.0f;
        for (int64_t at = threadIdx.x * V; at < c.dim; at += kLongBlock * V) {
            const int n = inside<V>(at, c.dim);
            load_weights<V>(w, weight, c.w_type, at, n, 1.0f);
            load_some_of<V>(v, from, at, n);
            load_some_of<V>(d, grad, at, n);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                first = first + d[k] * w[k];
                second = __builtin_fmaf(d[k] * w[k], (v[k] - mu) * r, second);
            }
        }
        row_sums<kLongBlock / kWave>(first, second, lds);
        first = first * each;
        second = second * each;
        for (int64_t at = threadIdx.x * V; at < c.dim; at += kLongBlock * V) {
            const int n = inside<V>(at, c.dim);
            float o[V];
            load_weights<V>(w, weight, c.w_type, at, n, 1.0f);
            load_some_of<V>(v, from, at, n);
            load_some_of<V>(d, grad, at, n);
            if (add) load_some_of<V>(o, add + row * c.x_stride, at, n);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float g = (d[k] * w[k] - first - (v[k] - mu) * r * second) * r;
                o[k] = add ? o[k] + g : g;
            }
            store_some_of<V>(dx + row * c.x_stride, at, o, n);
        }
    }
}

// The weights' terms of long rows: a workgroup's columns over a run of rows.
constexpr int kColumnBlock = 256;

template <class X, class Y>
__global__ void __launch_bounds__(kColumnBlock)
    norm_columns_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const float* mean, const float* rstd, float* partial,
                        int64_t run)
{
    constexpr int V = vec_of<X, Y>();
    const int64_t at = ((int64_t)blockIdx.x * kColumnBlock + threadIdx.x) * V;
    const int n = inside<V>(at, c.dim);
    if (n == 0) return;
    float dw[V] = {}, db[V] = {}, v[V], d[V];
    const int64_t end = (blockIdx.y + 1) * run < c.rows ? (blockIdx.y + 1) * run : c.rows;
    for (int64_t row = blockIdx.y * run; row < end; ++row) {
        const float mu = mean[row], r = rstd[row];
        load_some_of<V>(v, x + row * c.x_stride, at, n);
        load_some_of<V>(d, dy + row * c.y_stride, at, n);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            db[k] = db[k] + d[k];
            dw[k] = __builtin_fmaf(d[k], (v[k] - mu) * r, dw[k]);
        }
    }
    float* mine = partial + (int64_t)blockIdx.y * 2 * c.dim;
    store_some_of<V>(mine, at, dw, n);
    store_some_of<V>(mine + c.dim, at, db, n);
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
    if (at < 2 * dim) {
#pragma unroll 4
        for (int64_t k = lane; k < parts; k += kJoinRows) sum = sum + partial[k * 2 * dim + at];
    }
    lds[lane][col] = sum;
    __syncthreads();
    for (int half = kJoinRows / 2; half > 0; half /= 2) {
        if (lane < half) lds[lane][col] = lds[lane][col] + lds[lane + half][col];
        __syncthreads();
    }
    if (lane > 0 || at >= 2 * dim) return;
    void* to = at < dim ? dweight : dbias;
    const int64_t i = at < dim ? at : at - dim;
    if (!to) return;
    sum = lds[0][col];
    set_element_at(to, type, i, accumulate ? element_at(to, type, i) + sum : sum);
}

// ---- launches -----------------------------------------------------------------------

// Waves of a row, and vectors of V elements a lane holds of it.
struct Shape {
    int waves, k;
};

Shape shape_of(int64_t dim, int v)
{
    for (int waves = 1; waves <= 16; waves *= 4)
        for (int k = 1; k <= kHeldColumns / v; ++k)
            if (dim <= (int64_t)waves * kWave * k * v) return {waves, k};
    return {0, 0};
}

int vec_of_types(const ea_layer_norm_t& c)
{
    return c.x_type != EA_F32 && c.y_type != EA_F32 ? 8 : 4;
}

// f with the waves and vectors as constants.
template <int V, class F>
hipError_t with_shape(Shape s, F&& f)
{
#define EA_SHAPE(W, K) \
    if (s.waves == W && s.k == K) return f(std::integral_constant<int, W>{}, std::integral_constant<int, K>{})
    EA_SHAPE(1, 1);
    EA_SHAPE(1, 2);
    EA_SHAPE(4, 1);
    EA_SHAPE(4, 2);
    EA_SHAPE(16, 1);
    EA_SHAPE(16, 2);
    if constexpr (V == 4) {
        EA_SHAPE(1, 3);
        EA_SHAPE(1, 4);
        EA_SHAPE(4, 3);
        EA_SHAPE(4, 4);
        EA_SHAPE(16, 3);
        EA_SHAPE(16, 4);
    }
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
    return s.waves == 1 ? at_most((c.rows + 3) / 4, 1024) : at_most(c.rows, s.waves == 4 ? 1024 : 256);
}

// Runs of rows of long rows' column sums.
int64_t runs_of(const ea_layer_norm_t& c)
{
    return at_most((c.rows + 15) / 16, 64);
}

}  // namespace

int64_t layer_norm_workspace_bytes(const ea_layer_norm_t& c)
{
    const Shape s = shape_of(c.dim, vec_of_types(c));
    return (s.waves ? grad_groups_of(c, s) : runs_of(c)) * 2 * c.dim * 4;
}

hipError_t launch_layer_norm(const ea_layer_norm_t& c, const void* x, const void* weight, const void* bias, void* y,
                             float* mean, float* rstd, hipStream_t s)
{
    if (c.rows == 0) return hipSuccess;
    return with_type(c.x_type, [&](auto xt) {
        return with_type(c.y_type, [&](auto yt) {
            using X = decltype(xt);
            using Y = decltype(yt);
            const Shape shape = shape_of(c.dim, vec_of<X, Y>());
            if (!shape.waves) {
                hipLaunchKernelGGL((norm_long_kernel<X, Y>), dim3((unsigned)at_most(c.rows, 1024)), dim3(kLongBlock), 0,
                                   s, c, (const X*)x, weight, bias, (Y*)y, mean, rstd);
                return hipGetLastError();
            }
            const unsigned groups = (unsigned)norm_groups_of(c, shape);
            return with_shape<vec_of<X, Y>()>(shape, [&](auto w, auto k) {
                constexpr int W = decltype(w)::value, K = decltype(k)::value;
                hipLaunchKernelGGL((norm_kernel<X, Y, W, K>), dim3(groups), dim3(W == 1 ? 256 : W * kWave), 0, s, c,
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
    int64_t parts = 0;
    hipError_t e = hipSuccess;
    if (c.rows > 0)
        e = with_type(c.x_type, [&](auto xt) {
            return with_type(c.y_type, [&](auto yt) {
                using X = decltype(xt);
                using Y = decltype(yt);
                constexpr int V = vec_of<X, Y>();
                const Shape shape = shape_of(c.dim, V);
                if (!shape.waves) {
                    parts = runs_of(c);
                    const int64_t run = (c.rows + parts - 1) / parts;
                    const unsigned strips = (unsigned)((c.dim + kColumnBlock * V - 1) / (kColumnBlock * V));
                    // first: dx may take dy's place
                    if (partial)
                        hipLaunchKernelGGL((norm_columns_kernel<X, Y>), dim3(strips, (unsigned)parts),
                                           dim3(kColumnBlock), 0, s, c, (const X*)x, (const Y*)dy, mean, rstd, partial,
                                           run);
                    hipLaunchKernelGGL((norm_grad_long_kernel<X, Y>), dim3((unsigned)at_most(c.rows, 1024)),
                                       dim3(kLongBlock), 0, s, c, (const X*)x, (const Y*)dy, weight, mean, rstd,
                                       (const X*)add, (X*)dx);
                    return hipGetLastError();
                }
                parts = grad_groups_of(c, shape);
                return with_shape<V>(shape, [&](auto w, auto k) {
                    constexpr int W = decltype(w)::value, K = decltype(k)::value;
                    hipLaunchKernelGGL((norm_grad_kernel<X, Y, W, K>), dim3((unsigned)parts),
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
