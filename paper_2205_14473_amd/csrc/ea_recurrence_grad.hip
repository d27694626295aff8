// ea_recurrence_grad.hip -- the gradient of the gated linear recurrence (see
// ea_recurrence.hpp): the same tiles from the last to the first.  The state
// before each step is formed again from the states saved every 64 steps, so
// that g, x and dy are all that is read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_recurrence.hpp"

namespace ea {
namespace rec {

namespace {

// What arrives at step t from behind is e_t = a_{t+1} d_{t+1}, with d_t = dy_t + e_t; over some steps it goes from e to
// (product of their gates) e + (what they give from e = 0).

template <class X, class G, int C, bool SIGMOID>
__global__ void __launch_bounds__(kMostWaves* kWave)
    segment_grad_kernel(Call a, const G* g, const X* dy, const float* dh_last)
{
    __shared__ float lds[kMostWaves][2][kWave * C];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t each = a.c.batch * a.c.dim, units = a.p.strips * a.c.batch * a.p.segments;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const Place p = place_of<C>(a, unit);
        const int64_t stretch = a.p.steps / kMostWaves, row = p.b * a.c.length;
        float m[C], e[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            m[i] = 1.0f;
            e[i] = 0.0f;
        }
        for (int64_t t = p.from + (wave + 1) * stretch - kSteps; t >= p.from + wave * stretch; t -= kSteps) {
            const int count = steps_at(t, p.n);
            Vec<G, C> gr[kSteps];
            Vec<X, C> dr[kSteps];
            load_steps<C>(gr, g, row + t, a.c.g_stride, p, count);
            load_steps<C>(dr, dy, row + t, a.c.y_stride, p, count);
#pragma unroll
            for (int k = kSteps - 1; k >= 0; --k) {
                if (k < count) {
#pragma unroll
                    for (int i = 0; i < C; ++i) {
                        float f, w;
                        gate_of<SIGMOID>((float)element<C, G>(gr[k], i), f, w);
                        m[i] = m[i] * f;
                        e[i] = f * ((float)element<C, X>(dr[k], i) + e[i]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            lds[wave][0][lane * C + i] = m[i];
            lds[wave][1][lane * C + i] = e[i];
        }
        __syncthreads();
        if (wave == kMostWaves - 1) {
            for (int j = kMostWaves - 2; j >= 0; --j)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const float f = lds[j][0][lane * C + i];
                    m[i] = m[i] * f;
                    e[i] = behind(f, lds[j][1][lane * C + i], e[i]);
                }
            float* to = a.workspace + p.segment * 2 * each;
            store_floats<C>(to, p.b * a.c.dim + p.at, m, p.channels);
            store_floats<C>(to + each, p.b * a.c.dim + p.at, e, p.channels);
            if (p.segment == a.p.segments - 1) {       // dh0 may take dh_last's place
                load_floats<C>(e, dh_last, p.b * a.c.dim + p.at, p.channels);
                store_floats<C>(a.workspace + a.p.segments * 2 * each, p.b * a.c.dim + p.at, e, p.channels);
            }
        }
        __syncthreads();
    }
}

template <class X, class G, int C, bool SIGMOID>
__global__ void __launch_bounds__(kMostWaves* kWave)
    recurrence_grad_kernel(Call a, const G* g, const X* x, const float* states, const X* dy, const float* dh_last, G* dg,
                           X* dx, float* dh0)
{
    __shared__ Shared<C, 3> lds;
    const int wave = threadIdx.x / kWave, lane = lane_id(), waves = a.p.waves;
    const int64_t units = a.p.strips * a.c.batch * a.p.segments, tile = waves * kSteps;
    const int64_t blocks = (a.c.length + EA_RECURRENCE_BLOCK - 1) / EA_RECURRENCE_BLOCK;
    int parity = 0;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const Place p = place_of<C>(a, unit);
        const int64_t row = p.b * a.c.length;
        Vec<G, C> gr[kSteps];
        Vec<X, C> xr[kSteps], dr[kSteps];
        float saved[C];
        const int64_t tiles = (p.to - p.from + tile - 1) / tile;
        int64_t t = p.from + (tiles - 1) * tile + wave * kSteps;
        auto load = [&](int64_t t) {
            const int count = steps_at(t, p.n);
            load_steps<C>(gr, g, row + t, a.c.g_stride, p, count);
            load_steps<C>(xr, x, row + t, a.c.x_stride, p, count);
            load_steps<C>(dr, dy, row + t, a.c.y_stride, p, count);
            if (count > 0)
                load_floats<C>(saved, states, (p.b * blocks + t / EA_RECURRENCE_BLOCK) * a.c.dim + p.at, p.channels);
        };
        if (tiles > 0) load(t);
        float e[C];
        fold_segments<C, true>(e, a, p, dh_last);
        for (int64_t left = tiles; left > 0; --left, t -= tile) {
            const int count = steps_at(t, p.n);
            float f[kSteps * C], w[kSteps * C], u[kSteps * C], d[kSteps * C], h[C], m[C], end[C], back[C];
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int at = k * C + i;
                    gate_of<SIGMOID>((float)element<C, G>(gr[k], i), f[at], w[at]);
                    u[at] = (float)element<C, X>(xr[k], i);
                    d[at] = (float)element<C, X>(dr[k], i);
                    if (k >= count) {
                        f[at] = 1.0f;
                        w[at] = u[at] = d[at] = 0.0f;
                    }
                }
#pragma unroll
            for (int i = 0; i < C; ++i) {
                h[i] = count > 0 ? saved[i] : 0.0f;
                m[i] = 1.0f;
                end[i] = back[i] = 0.0f;
            }
            if (left > 1) load(t - tile);
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    m[i] = m[i] * f[k * C + i];
                    end[i] = __builtin_fmaf(f[k * C + i], end[i], w[k * C + i] * u[k * C + i]);
                }
#pragma unroll
            for (int k = kSteps - 1; k >= 0; --k)
#pragma unroll
                for (int i = 0; i < C; ++i) back[i] = f[k * C + i] * (d[k * C + i] + back[i]);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                lds.v[parity][wave][0][lane * C + i] = m[i];
                lds.v[parity][wave][1][lane * C + i] = end[i];
                lds.v[parity][wave][2][lane * C + i] = back[i];
            }
            __syncthreads();
            // the state before the wave's first step, from the saved one before it
            for (int j = wave / kGroupWaves * kGroupWaves; j < wave; ++j)
#pragma unroll
                for (int i = 0; i < C; ++i)
                    h[i] = behind(lds.v[parity][j][0][lane * C + i], lds.v[parity][j][1][lane * C + i], h[i]);
            float mine[C];
            for (int j = waves - 1; j >= 0; --j)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    if (j == wave) mine[i] = e[i];
                    e[i] = behind(lds.v[parity][j][0][lane * C + i], lds.v[parity][j][2][lane * C + i], e[i]);
                }
            parity ^= 1;
            float before[kSteps * C];
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    before[k * C + i] = h[i];
                    h[i] = __builtin_fmaf(f[k * C + i], h[i], w[k * C + i] * u[k * C + i]);
                }
#pragma unroll
            for (int k = kSteps - 1; k >= 0; --k) {
                float od[C], og[C];
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int at = k * C + i;
                    const float s = d[at] + mine[i];
                    mine[i] = f[at] * s;
                    od[i] = w[at] * s;
                    og[i] = SIGMOID ? s * (before[at] - u[at]) * (f[at] * w[at]) : s * before[at];
                    if (k >= count) {
                        mine[i] = s;
                        od[i] = og[i] = 0.0f;
                    }
                }
                if (t + k < p.to && p.channels > 0) {
                    X* tx = dx + (row + t + k) * a.c.x_stride + p.at;
                    G* tg = dg + (row + t + k) * a.c.g_stride + p.at;
                    if (p.channels == C) {
                        store_vec<C>(tx, narrow_from<C, X>(od));
                        store_vec<C>(tg, narrow_from<C, G>(og));
                    } else {
                        store_part<C>(tx, narrow_from<C, X>(od), p.channels);
                        store_part<C>(tg, narrow_from<C, G>(og), p.channels);
                    }
                }
            }
        }
        __syncthreads();                               // every wave has dh_last: dh0 may take its place
        if (dh0 && wave == 0 && p.segment == 0) store_floats<C>(dh0, p.b * a.c.dim + p.at, e, p.channels);
    }
}

}  // namespace
}  // namespace rec

hipError_t launch_recurrence_grad(const ea_recurrence_t& c, const void* g, const void* x, const float* states,
                                  const int32_t* lengths, const void* dy, const float* dh_last, void* dg, void* dx,
                                  float* dh0, void* workspace, hipStream_t s)
{
    using namespace rec;
    const int channels = channels_of(c, true);
    const Call a{c, plan_of(c, channels), lengths, (float*)workspace};
    const int64_t units = a.p.strips * c.batch * a.p.segments;
    if (units == 0) return hipSuccess;
    const unsigned groups = (unsigned)(units < kMostUnits ? units : kMostUnits);
    auto start = [&](auto xt, auto gt, auto ct, auto sigmoid) {
        using X = decltype(xt);
        using G = decltype(gt);
        constexpr int C = decltype(ct)::value;
        constexpr bool S = decltype(sigmoid)::value;
        if (a.p.segments > 1)
            hipLaunchKernelGGL((segment_grad_kernel<X, G, C, S>), dim3(groups), dim3(kMostWaves * kWave), 0, s, a,
                               (const G*)g, (const X*)dy, dh_last);
        hipLaunchKernelGGL((recurrence_grad_kernel<X, G, C, S>), dim3(groups), dim3(a.p.waves * kWave), 0, s, a,
                           (const G*)g, (const X*)x, states, (const X*)dy, dh_last, (G*)dg, (X*)dx, dh0);
        return hipGetLastError();
    };
    return with_type(c.x_type, [&](auto xt) {
        return with_type(c.g_type, [&](auto gt) {
            constexpr std::integral_constant<int, 1> one{};
            constexpr std::integral_constant<int, 2> two{};
            if (c.gate == EA_GATE_SIGMOID)
                return channels == 1 ? start(xt, gt, one, std::true_type{}) : start(xt, gt, two, std::true_type{});
            return channels == 1 ? start(xt, gt, one, std::false_type{}) : start(xt, gt, two, std::false_type{});
        });
    });
}

}  // namespace ea
