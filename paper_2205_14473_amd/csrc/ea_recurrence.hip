// ea_recurrence.hip -- the gated linear recurrence h_t = a_t h_{t-1} + w_t x_t
// over each channel of each sequence (see ea_recurrence.hpp).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_recurrence.hpp"

namespace ea {
namespace rec {

namespace {

// CHAIN: sequences of more than one chunk.  ONCE: y goes past the caches.
template <class X, class G, bool SIGMOID, bool CHAIN, bool ONCE>
__global__ void __launch_bounds__(kMostWaves* kWave, 8)
    recurrence_kernel(Call a, const G* g, const X* x, const float* h0, X* y, float* states, float* h_last)
{
    constexpr int K = kForwardSteps;
    __shared__ Exchange lds;
    const int wave = wave_id(), lane = lane_id(), waves = a.p.waves;
    const int64_t blocks = (a.c.length + EA_RECURRENCE_BLOCK - 1) / EA_RECURRENCE_BLOCK;
    for (Items<CHAIN> it(a, &lds.item); it.item < a.items;) {
        const Place p = place_of(a, it.item, false);
        it.draw(a);
        const int64_t t = (int64_t)(p.chunk * waves + wave) * K, row = p.b * a.c.length + t;
        const int count = steps_at<K>(t, p.n), held = steps_at<K>(t, (int)a.c.length);
        zero_steps<ONCE>(y, row, a.c.y_stride, a, p, count, held);
        if (p.chunk > p.last) {
            __syncthreads();
            it.next(a);
            __syncthreads();
            continue;
        }
        G gr[K];
        X xr[K];
        load_steps<K>(gr, g, row, a.c.g_stride, a, p, count);
        load_steps<K>(xr, x, row, a.c.x_stride, a, p, count);
        float f[K], v[K], m = 1.0f, e = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float w;
            gate_of<SIGMOID>((float)gr[k], f[k], w);
            v[k] = w * (float)xr[k];
        }
        mask_steps<K>(f, v, count);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            m = k ? m * f[k] : f[k];
            e = k ? __builtin_fmaf(f[k], e, v[k]) : f[k] * 0.0f + v[k];
        }
        lds.wave[wave][0][lane] = m;
        lds.wave[wave][1][lane] = e;
        const Link link = link_of(p, false);
        __syncthreads();
        it.next(a);
        float h;
        if (CHAIN) {
            meet<false>(a, p, link, lds, 1, h0);
            __syncthreads();
            h = fold_before(lds, link);
        } else {
            h = end_at(h0, a, p);
        }
#pragma unroll 4
        for (int j = 0; j < wave; ++j) h = behind(lds.wave[j][0][lane], lds.wave[j][1][lane], h);
        if (CHAIN && ends_stretch(link) && wave == waves - 1 && p.on)
            hand_out(stretch_word(a, p, link.stretch + 1), behind(m, e, h));
        if (states && p.on && t % EA_RECURRENCE_BLOCK == 0 && t < a.c.length)
            states[(p.b * blocks + t / EA_RECURRENCE_BLOCK) * a.c.dim + p.channel] = h;
        X* to = y + row * a.c.y_stride;
#pragma unroll
        for (int k = 0; k < K; ++k, to += a.c.y_stride) {
            h = __builtin_fmaf(f[k], h, v[k]);
            store_own<ONCE>(row_of(to, a, k < count), p, (X)h);
        }
        __syncthreads();                               // every wave has h0, and what is in LDS
        if (link.last && wave == waves - 1 && p.on) {
            if (h_last) h_last[p.b * a.c.dim + p.channel] = h;
            if (states)                                // of the chunks behind the last
                for (int64_t k = ((int64_t)(p.last + 1) * waves * K + EA_RECURRENCE_BLOCK - 1) / EA_RECURRENCE_BLOCK;
                     k < blocks; ++k)
                    states[(p.b * blocks + k) * a.c.dim + p.channel] = h;
        }
    }
}

constexpr int kClearBlock = 256;

// Workgroups of a launch: as many as the CUs hold where chunks are drawn from the counter.
constexpr int64_t kMostGroupsOf(bool chain)
{
    return chain ? 512 : 1 << 20;
}

__global__ void __launch_bounds__(kClearBlock) clear_kernel(uint64_t* words, int64_t count)
{
    typedef uint64_t Pair __attribute__((ext_vector_type(2)));
    for (int64_t i = (int64_t)blockIdx.x * kClearBlock + threadIdx.x; i * 2 < count;
         i += (int64_t)gridDim.x * kClearBlock)
        ((Pair*)words)[i] = Pair{0, 0};
}

}  // namespace

Plan plan_of(const ea_recurrence_t& c, int steps)
{
    Plan p;
    p.strips = (uint32_t)((c.dim + kWave - 1) / kWave);
    p.waves = 1;
    while (p.waves < kMostWaves && p.waves * steps < c.length) p.waves *= 2;
    const int64_t chunk = p.waves * steps;
    p.chunks = c.length > chunk ? (uint32_t)((c.length + chunk - 1) / chunk) : 1;
    p.groups = (p.chunks + kGroup - 1) / kGroup;
    return p;
}

// An even number: words are cleared in pairs.
int64_t words_of(const ea_recurrence_t& c, const Plan& p)
{
    if (p.chunks == 1) return 0;
    const int64_t pairs = (int64_t)p.chunks + p.groups, stretches = (p.groups + kGroup - 1) / kGroup;
    return (kCounterWords + (2 * pairs + stretches) * c.batch * c.dim + 1) / 2 * 2;
}

hipError_t begin(Call& a, const ea_recurrence_t& c, int steps, const int32_t* lengths, void* workspace,
                 unsigned* groups, hipStream_t s)
{
    a.c = c;
    a.p = plan_of(c, steps);
    a.lengths = lengths;
    a.words = (uint64_t*)workspace;
    *groups = 0;
    if (c.batch == 0) return hipSuccess;
    const int64_t items = (int64_t)a.p.strips * c.batch * a.p.chunks;
    a.items = (uint32_t)items;                         // under 2^31: checked with the configuration
    a.strips = Divisor(a.p.strips);
    a.batch = Divisor((uint32_t)c.batch);
    a.chunk = Divisor((uint32_t)(a.p.waves * steps));
    *groups = (unsigned)(items < kMostGroupsOf(a.p.chunks > 1) ? items : kMostGroupsOf(a.p.chunks > 1));
    if (a.p.chunks == 1) return hipSuccess;
    const int64_t count = words_of(c, a.p), clear = (count / 2 + kClearBlock - 1) / kClearBlock;
    hipLaunchKernelGGL(clear_kernel, dim3((unsigned)(clear < 2048 ? clear : 2048)), dim3(kClearBlock), 0, s, a.words,
                       count);
    return hipGetLastError();
}

}  // namespace rec

int64_t recurrence_workspace_bytes(const ea_recurrence_t& c)
{
    const int64_t forward = rec::words_of(c, rec::plan_of(c, rec::kForwardSteps));
    const int64_t backward = rec::words_of(c, rec::plan_of(c, rec::kBackwardSteps));
    return (forward > backward ? forward : backward) * 8;
}

hipError_t launch_recurrence(const ea_recurrence_t& c, const void* g, const void* x, const float* h0,
                             const int32_t* lengths, void* y, float* states, float* h_last, void* workspace,
                             hipStream_t s)
{
    using namespace rec;
    Call a;
    unsigned groups;
    const hipError_t e = begin(a, c, kForwardSteps, lengths, workspace, &groups, s);
    if (e != hipSuccess || groups == 0) return e;
    return with_kinds(c, [&](auto xt, auto gt, auto sigmoid) {
        using X = decltype(xt);
        using G = decltype(gt);
        constexpr bool S = decltype(sigmoid)::value;
        const dim3 grid(groups), block(a.p.waves * kWave);
        return with_bool(a.p.chunks > 1, [&](auto chain) {
            return with_bool(past_caches(c.batch * c.length * c.dim, c.x_type), [&](auto once) {
                hipLaunchKernelGGL((recurrence_kernel<X, G, S, decltype(chain)::value, decltype(once)::value>), grid,
                                   block, 0, s, a, (const G*)g, (const X*)x, h0, (X*)y, states, h_last);
                return hipGetLastError();
            });
        });
    });
}

}  // namespace ea
