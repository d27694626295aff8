// ea_recurrence_grad.hip -- the gradient of the gated linear recurrence (see
// ea_recurrence.hpp): the same chunks from the last to the first.  The state
// before each step is formed again from the states saved every 64 steps, so
// that g, x and dy are all that is read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_recurrence.hpp"

namespace ea {
namespace rec {

namespace {

// What arrives at step t from behind is e_t = a_{t+1} d_{t+1}, with d_t = dy_t + e_t; over some steps it goes from e to
// (product of their gates) e + (what they give from e = 0).  ONCE: dx and dg go past the caches.
template <class X, class G, bool SIGMOID, bool CHAIN, bool ONCE>
__global__ void __launch_bounds__(kMostWaves* kWave, 8)
    recurrence_grad_kernel(Call a, const G* g, const X* x, const float* states, const X* dy, const float* dh_last,
                           G* dg, X* dx, float* dh0)
{
    constexpr int K = kBackwardSteps, kBlockWaves = EA_RECURRENCE_BLOCK / K;
    __shared__ Exchange lds;
    const int wave = wave_id(), lane = lane_id(), waves = a.p.waves;
    const int64_t blocks = (a.c.length + EA_RECURRENCE_BLOCK - 1) / EA_RECURRENCE_BLOCK;
    for (Items<CHAIN> it(a, &lds.item); it.item < a.items;) {
        const Place p = place_of(a, it.item, true);
        it.draw(a);
        const int64_t t = (int64_t)(p.chunk * waves + wave) * K, row = p.b * a.c.length + t;
        const int count = steps_at<K>(t, p.n), held = steps_at<K>(t, (int)a.c.length);
        zero_steps<ONCE>(dx, row, a.c.x_stride, a, p, count, held);
        zero_steps<ONCE>(dg, row, a.c.g_stride, a, p, count, held);
        if (p.chunk > p.last) {
            __syncthreads();
            it.next(a);
            __syncthreads();
            continue;
        }
        G gr[K];
        X xr[K], dr[K];
        load_steps<K>(gr, g, row, a.c.g_stride, a, p, count);
        load_steps<K>(xr, x, row, a.c.x_stride, a, p, count);
        load_steps<K>(dr, dy, row, a.c.y_stride, a, p, count);
        float h = 0.0f;
        if (count > 0 && p.on) h = states[(p.b * blocks + t / EA_RECURRENCE_BLOCK) * a.c.dim + p.channel];
        float f[K], w[K], u[K], d[K], m = 1.0f, end = 0.0f, back = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            gate_of<SIGMOID>((float)gr[k], f[k], w[k]);
            u[k] = (float)xr[k];
            d[k] = (float)dr[k];
        }
        mask_steps<K>(f, u, count);
        mask_steps<K>(w, d, count);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            m = m * f[k];
            end = __builtin_fmaf(f[k], end, w[k] * u[k]);
        }
#pragma unroll
        for (int k = K - 1; k >= 0; --k) back = f[k] * (d[k] + back);
        lds.wave[wave][0][lane] = m;
        lds.wave[wave][1][lane] = end;
        lds.wave[wave][2][lane] = back;
        const Link link = link_of(p, true);
        __syncthreads();
        it.next(a);
        float e;
        if (CHAIN) {
            meet<true>(a, p, link, lds, 2, dh_last);
            __syncthreads();
            e = fold_before(lds, link);
        } else {
            e = end_at(dh_last, a, p);
        }
#pragma unroll 4
        for (int j = waves - 1; j > wave; --j) e = behind(lds.wave[j][0][lane], lds.wave[j][2][lane], e);
        if (CHAIN && ends_stretch(link) && wave == 0 && p.on)
            hand_out(stretch_word(a, p, link.stretch + 1), behind(m, back, e));
        // the state before the wave's first step, from the saved one before it
#pragma unroll 4
        for (int j = wave / kBlockWaves * kBlockWaves; j < wave; ++j)
            h = behind(lds.wave[j][0][lane], lds.wave[j][1][lane], h);
        // u becomes what the step's gradient is multiplied by for its gate
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float before = h;
            h = __builtin_fmaf(f[k], h, w[k] * u[k]);
            u[k] = SIGMOID ? (before - u[k]) * (f[k] * w[k]) : before;
        }
        X* tx = dx + (row + K - 1) * a.c.x_stride;
        G* tg = dg + (row + K - 1) * a.c.g_stride;
#pragma unroll
        for (int k = K - 1; k >= 0; --k, tx -= a.c.x_stride, tg -= a.c.g_stride) {
            const float s = d[k] + e;
            e = f[k] * s;                              // f = 1, d = 0 where the step does not count
            store_own<ONCE>(row_of(tx, a, k < count), p, (X)(w[k] * s));
            store_own<ONCE>(row_of(tg, a, k < count), p, (G)(u[k] * s));
        }
        __syncthreads();                               // every wave has dh_last, and what is in LDS
        if (link.last && wave == 0 && p.on && dh0) dh0[p.b * a.c.dim + p.channel] = e;
    }
}

}  // namespace
}  // namespace rec

hipError_t launch_recurrence_grad(const ea_recurrence_t& c, const void* g, const void* x, const float* states,
                                  const int32_t* lengths, const void* dy, const float* dh_last, void* dg, void* dx,
                                  float* dh0, void* workspace, hipStream_t s)
{
    using namespace rec;
    Call a;
    unsigned groups;
    const hipError_t status = begin(a, c, kBackwardSteps, lengths, workspace, &groups, s);
    if (status != hipSuccess || groups == 0) return status;
    return with_kinds(c, [&](auto xt, auto gt, auto sigmoid) {
        using X = decltype(xt);
        using G = decltype(gt);
        constexpr bool S = decltype(sigmoid)::value;
        const dim3 grid(groups), block(a.p.waves * kWave);
        return with_bool(a.p.chunks > 1, [&](auto chain) {
            return with_bool(past_caches(c.batch * c.length * c.dim, c.x_type), [&](auto once) {
                hipLaunchKernelGGL((recurrence_grad_kernel<X, G, S, decltype(chain)::value, decltype(once)::value>),
                                   grid, block, 0, s, a, (const G*)g, (const X*)x, states, (const X*)dy, dh_last,
                                   (G*)dg, (X*)dx, dh0);
                return hipGetLastError();
            });
        });
    });
}

}  // namespace ea
