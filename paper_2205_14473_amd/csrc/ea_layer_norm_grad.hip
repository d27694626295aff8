// ea_layer_norm_grad.hip -- the gradient of layer norm.
//
// Rows are held as in the forward pass.  The gradient of the weights is a sum over
// rows: each workgroup adds its rows' terms in registers and leaves one partial
// row, and a second launch adds those.  Which rows a workgroup takes depends on
// the sizes alone, so every sum has one order.
//
// Bound by bytes: 65,536 x 1,024 bfloat16 with a residual's gradient added 103 us,
// 5.2 TB/s, of which the partial rows' sum is 6; 4,096 x 16,384 115 us, 4.7 TB/s.  Few
// rows are bound by the two launches: 2,048 x 768 binary32 12 us.  Rows that are not
// held read x and dy three times: 2,048 x 20,000 bfloat16 117 us, 2.8 TB/s of what
// they have to move (the norm itself, three times x: 42 us, 3.9).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_layer_norm.hpp"

namespace ea {
namespace norm {

namespace {

// Floats of a partial row of dweight, and of dbias behind it: whole vectors, what lies behind the columns is not looked
// at.
__host__ __device__ constexpr int64_t partial_row(int64_t dim)
{
    return (dim + 7) / 8 * 8;
}

// Whether the next row's vectors are asked for before this row's sums are formed, `add` in all of these.  The registers for
// them pay where a lane holds few columns (131,072 x 256 bfloat16 66 us without, 55 with) and for rows with a tail, whose
// loads are more and smaller (65,536 x 1,001 121 without, 104 with); not for 16 whole columns a lane (32,768 x 1,024
// binary32 102 without, 107 with; 65,536 x 1,024 bfloat16 103 either way), nor for 16 waves, which have 128 registers each
// (4,096 x 16,384 bfloat16 115 without, 130 with; binary32 218 and 349).
constexpr bool grad_ahead(int waves, int columns, bool tail)
{
    return waves <= 4 && (columns <= 8 || tail);
}

// Waves of a SIMD that the gradient's registers leave room for (four and spills for 1,001 columns: 230 us).  Forms of 16
// columns a lane with a binary32 array still keep 4 to 16 registers in scratch, of 16 waves with a tail and arrays of two
// sizes 41 to 59.
constexpr int grad_waves(int waves, int columns, bool tail)
{
    return grad_ahead(waves, columns, tail) && columns > 8 ? 3 : 4;
}

// n, each: dim and 1 / dim, from the host so that they are scalars.  The means are subtracted, and what they leave is
// multiplied by rstd: they are quotients, so that they leave nothing where the sums are exact.  ONCE: the result goes past
// the caches.
template <class X, class Y, bool TAIL, int WAVES, int K, bool ONCE>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave, (grad_waves(WAVES, K * kVec<X, Y, TAIL>, TAIL)))
    norm_grad_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const void* weight, const float* mean,
                     const float* rstd, const X* add, X* dx, float* partial, float n, float each)
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
        // (scalars: in vector registers 16-wave rows spill a hundred others, 4,096 x 16,384 bfloat16 150 us, and 115 so)
        first = uniform(quotient(first, n, each));
        second = uniform(quotient(second, n, each));
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
            store_row<V, ONCE>(dx + row * c.x_stride, at, o, dim, tail);
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

template <class X, class Y, bool TAIL, bool ONCE>
__global__ void __launch_bounds__(kLongBlock)
    norm_grad_long_kernel(ea_layer_norm_t c, const X* x, const Y* dy, const void* weight, const float* mean,
                          const float* rstd, const X* add, X* dx, float n, float each)
{
    constexpr int V = vec_of<X, Y, TAIL>();
    __shared__ float2 lds[kLongBlock / kWave];
    const int dim = (int)c.dim;
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
        first = uniform(quotient(first, n, each));
        second = uniform(quotient(second, n, each));
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
            store_row<V, ONCE>(dx + row * c.x_stride, at, o, dim, TAIL);
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

// Workgroups of a launch.
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
}  // namespace norm

int64_t layer_norm_workspace_bytes(const ea_layer_norm_t& c)
{
    using namespace norm;
    const Shape s = shape_of(c);
    return (s.waves ? grad_groups_of(c, s) : runs_of(c)) * 2 * partial_row(c.dim) * 4;
}

hipError_t launch_layer_norm_grad(const ea_layer_norm_t& c, const void* x, const void* dy, const void* weight,
                                  const float* mean, const float* rstd, const void* add, void* dx, void* dweight,
                                  void* dbias, bool accumulate, void* workspace, hipStream_t s)
{
    using namespace norm;
    float* partial = dweight || dbias ? (float*)workspace : nullptr;
    const Shape shape = shape_of(c);
    const int64_t parts = c.rows == 0 ? 0 : shape.waves ? grad_groups_of(c, shape) : runs_of(c);
    const float n = (float)c.dim, each = 1.0f / n;
    hipError_t e = hipSuccess;
    if (c.rows > 0)
        e = with_type(c.x_type, [&](auto xt) {
            return with_type(c.y_type, [&](auto yt) {
                return with_bool(past_caches(c.rows * c.dim, c.x_type), [&](auto once) {
                    constexpr bool O = decltype(once)::value;
                    using X = decltype(xt);
                    using Y = decltype(yt);
                    if (!shape.waves) {
                        const int64_t run = (c.rows + parts - 1) / parts;
                        const int64_t strip = kColumnBlock * (shape.tail ? 4 : vec_of<X, Y, false>());
                        auto* columns = shape.tail ? norm_columns_kernel<X, Y, true> : norm_columns_kernel<X, Y, false>;
                        auto* rows =
                            shape.tail ? norm_grad_long_kernel<X, Y, true, O> : norm_grad_long_kernel<X, Y, false, O>;
                        // first: dx may take dy's place
                        if (partial)
                            hipLaunchKernelGGL(columns, dim3((unsigned)((c.dim + strip - 1) / strip), (unsigned)parts),
                                               dim3(kColumnBlock), 0, s, c, (const X*)x, (const Y*)dy, mean, rstd,
                                               partial, run);
                        hipLaunchKernelGGL(rows, dim3((unsigned)at_most(c.rows, 1024)), dim3(kLongBlock), 0, s, c,
                                           (const X*)x, (const Y*)dy, weight, mean, rstd, (const X*)add, (X*)dx, n,
                                           each);
                        return hipGetLastError();
                    }
                    return with_shape<vec_of<X, Y, false>()>(shape, [&](auto t, auto w, auto k) {
                        constexpr int W = decltype(w)::value, K = decltype(k)::value;
                        constexpr bool T = decltype(t)::value;
                        hipLaunchKernelGGL((norm_grad_kernel<X, Y, T, W, K, O>), dim3((unsigned)parts),
                                           dim3(W == 1 ? 256 : W * kWave), 0, s, c, (const X*)x, (const Y*)dy, weight,
                                           mean, rstd, (const X*)add, (X*)dx, partial, n, each);
                        return hipGetLastError();
                    });
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
