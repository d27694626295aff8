// ea_recurrence.hip -- the gated linear recurrence h_t = a_t h_{t-1} + w_t x_t
// over each channel of each sequence (see ea_recurrence.hpp).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_recurrence.hpp"

namespace ea {
namespace rec {

namespace {

// A segment's product of gates and the state it ends with from 0: each wave runs over a stretch of consecutive steps.
template <class X, class G, int C, bool SIGMOID>
__global__ void __launch_bounds__(kMostWaves* kWave) segment_kernel(Call a, const G* g, const X* x, const float* h0)
{
    __shared__ float lds[kMostWaves][2][kWave * C];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t each = a.c.batch * a.c.dim, units = a.p.strips * a.c.batch * a.p.segments;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const Place p = place_of<C>(a, unit);
        const int64_t stretch = a.p.steps / kMostWaves, row = p.b * a.c.length;
        float m[C], h[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            m[i] = 1.0f;
            h[i] = 0.0f;
        }
        for (int64_t t = p.from + wave * stretch; t < p.from + (wave + 1) * stretch; t += kSteps) {
            const int count = steps_at(t, p.n);
            Vec<G, C> gr[kSteps];
            Vec<X, C> xr[kSteps];
            load_steps<C>(gr, g, row + t, a.c.g_stride, p, count);
            load_steps<C>(xr, x, row + t, a.c.x_stride, p, count);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                if (k >= count) break;
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    float f, w;
                    gate_of<SIGMOID>((float)element<C, G>(gr[k], i), f, w);
                    m[i] = m[i] * f;
                    h[i] = __builtin_fmaf(f, h[i], w * (float)element<C, X>(xr[k], i));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            lds[wave][0][lane * C + i] = m[i];
            lds[wave][1][lane * C + i] = h[i];
        }
        __syncthreads();
        if (wave == 0) {
            for (int j = 1; j < kMostWaves; ++j)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const float f = lds[j][0][lane * C + i];
                    m[i] = m[i] * f;
                    h[i] = behind(f, lds[j][1][lane * C + i], h[i]);
                }
            float* to = a.workspace + p.segment * 2 * each;
            store_floats<C>(to, p.b * a.c.dim + p.at, m, p.channels);
            store_floats<C>(to + each, p.b * a.c.dim + p.at, h, p.channels);
            if (p.segment == 0) {                      // h_last may take h0's place
                load_floats<C>(h, h0, p.b * a.c.dim + p.at, p.channels);
                store_floats<C>(a.workspace + a.p.segments * 2 * each, p.b * a.c.dim + p.at, h, p.channels);
            }
        }
        __syncthreads();
    }
}

template <class X, class G, int C, bool SIGMOID>
__global__ void __launch_bounds__(kMostWaves* kWave)
    recurrence_kernel(Call a, const G* g, const X* x, const float* h0, X* y, float* states, float* h_last)
{
    __shared__ Shared<C, 2> lds;
    const int wave = threadIdx.x / kWave, lane = lane_id(), waves = a.p.waves;
    const int64_t units = a.p.strips * a.c.batch * a.p.segments, tile = waves * kSteps;
    const int64_t blocks = (a.c.length + EA_RECURRENCE_BLOCK - 1) / EA_RECURRENCE_BLOCK;
    int parity = 0;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const Place p = place_of<C>(a, unit);
        const int64_t row = p.b * a.c.length;
        Vec<G, C> gr[kSteps];
        Vec<X, C> xr[kSteps];
        int64_t t = p.from + wave * kSteps;
        load_steps<C>(gr, g, row + t, a.c.g_stride, p, steps_at(t, p.n));
        load_steps<C>(xr, x, row + t, a.c.x_stride, p, steps_at(t, p.n));
        float h[C];
        fold_segments<C, false>(h, a, p, h0);
        for (; t - wave * kSteps < p.to; t += tile) {
            const int count = steps_at(t, p.n);
            float f[kSteps * C], v[kSteps * C], m[C], e[C];
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    float w;
                    gate_of<SIGMOID>((float)element<C, G>(gr[k], i), f[k * C + i], w);
                    v[k * C + i] = w * (float)element<C, X>(xr[k], i);
                    if (k >= count) {
                        f[k * C + i] = 1.0f;
                        v[k * C + i] = 0.0f;
                    }
                }
            if (t + tile - wave * kSteps < p.to) {     // the next tile's steps, while this one's are worked on
                const int next = steps_at(t + tile, p.n);
                load_steps<C>(gr, g, row + t + tile, a.c.g_stride, p, next);
                load_steps<C>(xr, x, row + t + tile, a.c.x_stride, p, next);
            }
#pragma unroll
            for (int i = 0; i < C; ++i) {
                m[i] = f[i];
                e[i] = v[i];
            }
#pragma unroll
            for (int k = 1; k < kSteps; ++k)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    m[i] = m[i] * f[k * C + i];
                    e[i] = __builtin_fmaf(f[k * C + i], e[i], v[k * C + i]);
                }
#pragma unroll
            for (int i = 0; i < C; ++i) {
                lds.v[parity][wave][0][lane * C + i] = m[i];
                lds.v[parity][wave][1][lane * C + i] = e[i];
            }
            __syncthreads();
            float mine[C];
            for (int j = 0; j < waves; ++j)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    if (j == wave) mine[i] = h[i];
                    h[i] = behind(lds.v[parity][j][0][lane * C + i], lds.v[parity][j][1][lane * C + i], h[i]);
                }
            parity ^= 1;
            if (states && t % EA_RECURRENCE_BLOCK == 0 && t < p.to)
                store_floats<C>(states, (p.b * blocks + t / EA_RECURRENCE_BLOCK) * a.c.dim + p.at, mine, p.channels);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                if (t + k >= p.to) break;
                float o[C];
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    mine[i] = __builtin_fmaf(f[k * C + i], mine[i], v[k * C + i]);
                    o[i] = k < count ? mine[i] : 0.0f;
                }
                X* to = y + (row + t + k) * a.c.y_stride + p.at;
                if (p.channels == C)
                    store_vec<C>(to, narrow_from<C, X>(o));
                else
                    store_part<C>(to, narrow_from<C, X>(o), p.channels);
            }
        }
        __syncthreads();                               // every wave has h0: h_last may take its place
        if (h_last && wave == 0 && p.segment == a.p.segments - 1)
            store_floats<C>(h_last, p.b * a.c.dim + p.at, h, p.channels);
    }
}

}  // namespace

int channels_of(const ea_recurrence_t& c, bool backward)
{
    if (c.dim <= kWave) return 1;
    if (backward) return c.x_type != EA_F32 && c.g_type != EA_F32 ? 2 : 1;
    return 2;
}

Plan plan_of(const ea_recurrence_t& c, int channels)
{
    Plan p;
    p.strips = (c.dim + kWave * channels - 1) / (kWave * channels);
    p.waves = 1;
    while (p.waves < kMostWaves && p.waves * kSteps < c.length) p.waves *= 2;
    p.segments = 1;
    p.steps = (c.length + kTile - 1) / kTile * kTile;
    const int64_t units = p.strips * c.batch;
    if (units > 0 && units < 192 && c.length > 4 * kTile) {
        int64_t want = (512 + units - 1) / units;
        const int64_t tiles = (c.length + kTile - 1) / kTile;
        if (want > tiles / 2) want = tiles / 2;
        const int64_t each = (tiles + want - 1) / want;
        p.segments = (tiles + each - 1) / each;
        p.steps = each * kTile;
    }
    return p;
}

}  // namespace rec

int64_t recurrence_workspace_bytes(const ea_recurrence_t& c)
{
    int64_t most = 0;
    for (const bool backward : {false, true}) {
        const int64_t n = rec::plan_of(c, rec::channels_of(c, backward)).segments;
        most = n > most ? n : most;
    }
    return most > 1 ? (2 * most + 1) * c.batch * c.dim * 4 : 0;
}

hipError_t launch_recurrence(const ea_recurrence_t& c, const void* g, const void* x, const float* h0,
                             const int32_t* lengths, void* y, float* states, float* h_last, void* workspace,
                             hipStream_t s)
{
    using namespace rec;
    const int channels = channels_of(c, false);
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
            hipLaunchKernelGGL((segment_kernel<X, G, C, S>), dim3(groups), dim3(kMostWaves * kWave), 0, s, a,
                               (const G*)g, (const X*)x, h0);
        hipLaunchKernelGGL((recurrence_kernel<X, G, C, S>), dim3(groups), dim3(a.p.waves * kWave), 0, s, a,
                           (const G*)g, (const X*)x, h0, (X*)y, states, h_last);
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
