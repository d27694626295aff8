// ea_layer_norm.hip -- layer norm.
//
// A row is held in registers by 1, 4 or 16 waves, 16 elements a lane at most,
// so that every array passes memory once; rows of more than 16,384 columns are
// read again for each of their sums.
//
// The squares are summed of differences from the mean, from the same registers:
// nothing cancels.  The mean is a quotient, not a product with a rounded 1 / dim: a row
// of one value whose sum is exact has that value as its mean, and gives the bias (as a
// product the mean is a unit off at some widths, and 1 / sqrt(eps) times that is in the
// result: up to 0.3 for a row of 10,000s).
//
// Bound by bytes: 65,536 x 1,024 bfloat16 50 us, 5.4 TB/s, where a copy of as much
// reaches 5.1.  Few rows are bound by the launch: 16 x 768 3 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_layer_norm.hpp"

namespace ea {
namespace norm {

namespace {

template <int WAVES>
__device__ __forceinline__ float row_sum(float a, float2* lds)
{
    float none = 0.0f;
    if (WAVES == 1) return wave_sum(a);
    row_sums<WAVES>(a, none, lds);
    return a;
}

// n, each: dim and 1 / dim, from the host so that they are scalars (in vector registers one wave less fits a SIMD: 65,536
// x 1,024 bfloat16 52.7 us, and 50.2 this way).  ONCE: the result goes past the caches.
template <class X, class Y, bool TAIL, int WAVES, int K, bool ONCE>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave)
    norm_kernel(ea_layer_norm_t c, const X* x, const void* weight, const void* bias, Y* y, float* mean, float* rstd,
                float n, float each)
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
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave_id() : 0); row < c.rows;
         row += (int64_t)gridDim.x * kRows) {
        float v[K * V], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            load_row<V>(v + k * V, x + row * c.x_stride, (k * WAVES * kWave + lane) * V, dim,
                        tail_of<TAIL, WAVES, K>(k));
#pragma unroll
        for (int k = 0; k < K * V; ++k) sum = sum + v[k];
        const float mu = quotient(row_sum<WAVES>(sum, lds), n, each);
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
            store_row<V, ONCE>(y + row * c.y_stride, (k * WAVES * kWave + lane) * V, v + k * V, dim,
                               tail_of<TAIL, WAVES, K>(k));
        if (lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

// Rows too long to hold: a workgroup a row, read once for each sum and once more.
template <class X, class Y, bool TAIL, bool ONCE>
__global__ void __launch_bounds__(kLongBlock)
    norm_long_kernel(ea_layer_norm_t c, const X* x, const void* weight, const void* bias, Y* y, float* mean,
                     float* rstd, float n, float each)
{
    constexpr int V = vec_of<X, Y, TAIL>();
    __shared__ float2 lds[kLongBlock / kWave];
    const int dim = (int)c.dim;
    for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
        const X* from = x + row * c.x_stride;
        Y* to = y + row * c.y_stride;
        float v[V], sum = 0.0f, squares = 0.0f;
        for (int at = threadIdx.x * V; at < dim; at += kLongBlock * V) {
            load_row<V>(v, from, at, dim, TAIL ? kTail : 0);
#pragma unroll
            for (int k = 0; k < V; ++k) sum = sum + v[k];
        }
        const float mu = quotient(row_sum<kLongBlock / kWave>(sum, lds), n, each);
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
            store_row<V, ONCE>(to, at, v, dim, TAIL);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

// Workgroups of a launch.
int64_t norm_groups_of(const ea_layer_norm_t& c, Shape s)
{
    return s.waves == 1 ? at_most((c.rows + 3) / 4, 2048) : at_most(c.rows, s.waves == 4 ? 2048 : 512);
}

}  // namespace
}  // namespace norm

hipError_t launch_layer_norm(const ea_layer_norm_t& c, const void* x, const void* weight, const void* bias, void* y,
                             float* mean, float* rstd, hipStream_t s)
{
    using namespace norm;
    if (c.rows == 0) return hipSuccess;
    const Shape shape = shape_of(c);
    const float n = (float)c.dim, each = 1.0f / n;
    return with_type(c.x_type, [&](auto xt) {
        return with_type(c.y_type, [&](auto yt) {
            return with_bool(past_caches(c.rows * c.dim, c.y_type), [&](auto once) {
                using X = decltype(xt);
                using Y = decltype(yt);
                constexpr bool O = decltype(once)::value;
                if (!shape.waves) {
                    auto* kernel = shape.tail ? norm_long_kernel<X, Y, true, O> : norm_long_kernel<X, Y, false, O>;
                    hipLaunchKernelGGL(kernel, dim3((unsigned)at_most(c.rows, 1024)), dim3(kLongBlock), 0, s, c,
                                       (const X*)x, weight, bias, (Y*)y, mean, rstd, n, each);
                    return hipGetLastError();
                }
                const unsigned groups = (unsigned)norm_groups_of(c, shape);
                return with_shape<vec_of<X, Y, false>()>(shape, [&](auto t, auto w, auto k) {
                    constexpr int W = decltype(w)::value, K = decltype(k)::value;
                    constexpr bool T = decltype(t)::value;
                    hipLaunchKernelGGL((norm_kernel<X, Y, T, W, K, O>), dim3(groups),
                                       dim3(W == 1 ? 256 : W * kWave), 0, s, c, (const X*)x, weight, bias, (Y*)y, mean,
                                       rstd, n, each);
                    return hipGetLastError();
                });
            });
        });
    });
}

}  // namespace ea
