// ea_dropout.hip -- dropout from the library's counter-based draws, with a
// residual added, and its gradient: one pass, nothing stored but the result.
//
// A thread takes the eight elements that one application of Philox4x32-10 has
// 16-bit draws for.  The draws are numbered by the element's row and column
// alone, so strides, types and the launch do not change which are dropped.
//
// Bound by bytes: with draws of 16 bits an application's forty multiplications serve
// eight elements.  50,003 x 1,001 binary16: 34 us for the gradient, 5.9 TB/s; 2,048 x
// 768 binary32 with the residual: 5 us, most of it the launch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "ea_layer.hpp"

namespace ea {

namespace {

constexpr int kDropBlock = 256;
constexpr int kDraws = 8;                              // of one application
constexpr int64_t kMostDropGroups = 1 << 22;           // workgroups of a launch: a grid has fewer than 2^32 threads

struct Drop {
    int64_t total;                                     // elements
    int64_t dim;                                       // columns (of rows with gaps)
    int64_t in_stride, out_stride;
    uint32_t limit;                                    // draws under it are dropped
    float factor;
    uint32_t t, site, k0, k1;
    const uint32_t* t_dev;
};

template <class A, class B>
__device__ __forceinline__ float dropped(const Drop& c, A x, B residual, bool add, uint32_t word, int half)
{
    const uint32_t u = half ? word >> 16 : word & 0xFFFFu;
    const float v = u >= c.limit ? (float)x * c.factor : 0.0f;
    return add ? (float)residual + v : v;
}

// A: type read, B: type written and of the residual.  DENSE: no elements between rows, so element n lies at n.
// ONCE: the result goes past the caches.
template <class A, class B, bool DENSE, bool ONCE>
__global__ void __launch_bounds__(kDropBlock) dropout_kernel(Drop c, const A* in, const B* residual, B* out)
{
    const uint32_t t = c.t_dev ? *c.t_dev : c.t;
    for (int64_t group = (int64_t)blockIdx.x * kDropBlock + threadIdx.x; group * kDraws < c.total;
         group += (int64_t)gridDim.x * kDropBlock) {
        const int64_t first = group * kDraws;
        const uint4 r = philox10(make_uint4((uint32_t)group, (uint32_t)((uint64_t)group >> 32), t, c.site), c.k0, c.k1);
        const uint32_t word[4] = {r.x, r.y, r.z, r.w};
        const int left = c.total - first < kDraws ? (int)(c.total - first) : kDraws;
        int64_t row = 0, col = first;
        if (!DENSE) {
            row = first / c.dim;
            col = first - row * c.dim;
        }
        if (left == kDraws && (DENSE || c.dim - col >= kDraws)) {
            const int64_t to = row * c.out_stride + col;
            const Vec<A, 8> x = load_vec<8>(in + row * c.in_stride + col);
            Vec<B, 8> res = {}, y;
            if (residual) res = load_vec<8>(residual + to);
#pragma unroll
            for (int k = 0; k < kDraws; ++k)
                y[k] = (B)dropped(c, x[k], res[k], residual != nullptr, word[k / 2], k & 1);
            store_vec<8, ONCE>(out + to, y);
            continue;
        }
#pragma unroll
        for (int k = 0; k < kDraws; ++k) {
            if (k < left) {
                const int64_t to = row * c.out_stride + col;
                const B res = residual ? residual[to] : (B)0.0f;
                out[to] = (B)dropped(c, in[row * c.in_stride + col], res, residual != nullptr, word[k / 2], k & 1);
                if (++col == c.dim && !DENSE) {
                    col = 0;
                    ++row;
                }
            }
        }
    }
}

}  // namespace

hipError_t launch_dropout(const ea_dropout_t& c, bool backward, uint32_t t, const uint32_t* t_dev, const void* in,
                          const void* residual, void* out, hipStream_t s)
{
    Drop d{};
    d.total = c.rows * c.dim;
    if (d.total == 0) return hipSuccess;
    d.dim = c.dim;
    d.in_stride = backward ? c.y_stride : c.x_stride;
    d.out_stride = backward ? c.x_stride : c.y_stride;
    d.limit = (uint32_t)std::nearbyint((double)c.p * 65536.0);
    d.factor = d.limit < 65536 ? (float)(65536.0 / (65536.0 - d.limit)) : 0.0f;
    d.t = t;
    d.t_dev = t_dev;
    d.site = c.site;
    d.k0 = (uint32_t)c.seed;
    d.k1 = (uint32_t)(c.seed >> 32);
    const bool dense = c.rows == 1 || (c.x_stride == c.dim && c.y_stride == c.dim);
    const int64_t groups = (d.total + kDraws - 1) / kDraws, most = kMostDropGroups;
    const int64_t blocks = groups < most * kDropBlock ? (groups + kDropBlock - 1) / kDropBlock : most;
    return with_type(backward ? c.y_type : c.x_type, [&](auto a) {
        return with_type(backward ? c.x_type : c.y_type, [&](auto b) {
            using A = decltype(a);
            using B = decltype(b);
            return with_bool(dense, [&](auto packed) {
                return with_bool(past_caches(d.total, backward ? c.x_type : c.y_type), [&](auto once) {
                    hipLaunchKernelGGL((dropout_kernel<A, B, decltype(packed)::value, decltype(once)::value>),
                                       dim3((unsigned)blocks), dim3(kDropBlock), 0, s, d, (const A*)in,
                                       (const B*)residual, (B*)out);
                    return hipGetLastError();
                });
            });
        });
    });
}

}  // namespace ea
