// ea_recurrence.hpp -- what the gated linear recurrence and its gradient share:
// the plan of a call, gates, loads of a wave's steps.
//
// A workgroup takes 64 * C channels of one sequence, C a lane, and walks over
// tiles of steps: each of its waves takes kSteps consecutive steps of a tile,
// reads them ahead of the tile before, and runs them from a state of 0; the
// product of their gates and the state they end with go to LDS, and after one
// barrier every wave folds what lies before it, in order, and runs its steps
// again from the true state.  Where there are too few channels to fill the GPU
// a sequence is cut into segments: a first launch leaves each segment's product
// and end state, and every segment's workgroup folds those before it.
#pragma once

#include "ea_layer.hpp"

namespace ea {
namespace rec {

constexpr int kSteps = 8;                              // of a wave and tile
constexpr int kMostWaves = 16;
constexpr int kTile = kSteps * kMostWaves;             // steps of a tile of a sequence that is longer than one
constexpr int kGroupWaves = EA_RECURRENCE_BLOCK / kSteps;   // waves between two saved states

struct Plan {
    int64_t strips;                                    // of 64 * C channels
    int64_t segments, steps;                           // of a sequence, and steps of each (a multiple of kTile)
    int waves;
};

struct Call {
    ea_recurrence_t c;
    Plan p;
    const int32_t* lengths;
    float* workspace;                                  // [segments][2][batch * dim], then [batch * dim]: the start
};

// The part of the work that workgroup `unit` has: its channels' strip, sequence and segment.
struct Place {
    int64_t b, segment;
    int64_t at;                                        // the lane's first channel
    int channels;                                      // it has, 0 to C
    int64_t n;                                         // steps of the sequence that count
    int64_t from, to;                                  // the segment's steps
};

template <int C>
__device__ __forceinline__ Place place_of(const Call& a, int64_t unit)
{
    Place p;
    const int64_t strip = unit % a.p.strips, rest = unit / a.p.strips;
    p.b = rest % a.c.batch;
    p.segment = rest / a.c.batch;
    p.at = (strip * kWave + lane_id()) * C;
    const int64_t left = a.c.dim - p.at;
    p.channels = left >= C ? C : left > 0 ? (int)left : 0;
    p.n = a.c.length;
    if (a.lengths) {
        const int64_t n = a.lengths[p.b];
        p.n = n < 0 ? 0 : n < p.n ? n : p.n;
    }
    p.from = p.segment * a.p.steps;
    p.to = p.from + a.p.steps < a.c.length ? p.from + a.p.steps : a.c.length;
    return p;
}

// The first `count` of a wave's steps from row `row` on, as they are stored; the others are left unset.
template <int C, class T>
__device__ __forceinline__ void load_steps(Vec<T, C>* v, const T* p, int64_t row, int64_t stride, const Place& at, int count)
{
    if (at.channels == 0) return;
    const T* from = p + row * stride + at.at;
    if (at.channels == C && count == kSteps) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) v[k] = load_vec<C>(from + k * stride);
        return;
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
        if (k < count) v[k] = load_part<C>(from + k * stride, at.channels);
}

// Steps of the wave at step `t` that count, 0 to kSteps.
__device__ __forceinline__ int steps_at(int64_t t, int64_t n)
{
    const int64_t left = n - t;
    return left >= kSteps ? kSteps : left > 0 ? (int)left : 0;
}

// a and w of a gate: 1 / (1 + e) and e / (1 + e) with e = exp(-|g|).  The reciprocal gets a correction step: gates near
// 1 are multiplied over hundreds of steps, where a unit each would add up.
template <bool SIGMOID>
__device__ __forceinline__ void gate_of(float g, float& a, float& w)
{
    if (!SIGMOID) {
        a = g;
        w = 1.0f;
        return;
    }
    const float e = __builtin_amdgcn_exp2f(-fabsf(g) * 0x1.715476p+0f);
    const float d = 1.0f + e, q = __builtin_amdgcn_rcpf(d);
    const float r = __builtin_fmaf(__builtin_fmaf(-d, q, 1.0f), q, q), s = e * r;
    a = g < 0.0f ? s : r;
    w = g < 0.0f ? r : s;
}

// h behind steps whose gates' product is a and that lead from 0 to v.  A state of 0 stays out of the product: gates
// that multiply to infinity leave it what the steps one by one would.
__device__ __forceinline__ float behind(float a, float v, float h)
{
    return h == 0.0f ? v : __builtin_fmaf(a, h, v);
}

template <int C>
__device__ __forceinline__ void load_floats(float* x, const float* p, int64_t at, int channels)
{
#pragma unroll
    for (int k = 0; k < C; ++k) x[k] = p && k < channels ? p[at + k] : 0.0f;
}

template <int C>
__device__ __forceinline__ void store_floats(float* p, int64_t at, const float* x, int channels)
{
#pragma unroll
    for (int k = 0; k < C; ++k)
        if (k < channels) p[at + k] = x[k];
}

// The state (or gradient) that segment `p.segment` starts with: the ones before it (or behind, from the last) folded.
template <int C, bool REVERSE>
__device__ __forceinline__ void fold_segments(float* h, const Call& a, const Place& p, const float* start)
{
    const int64_t each = a.c.batch * a.c.dim, at = p.b * a.c.dim + p.at;
    if (a.p.segments == 1) {
        load_floats<C>(h, start, at, p.channels);
        return;
    }
    load_floats<C>(h, a.workspace + a.p.segments * 2 * each, at, p.channels);
    const int64_t count = REVERSE ? a.p.segments - 1 - p.segment : p.segment;
#pragma unroll 4
    for (int64_t i = 0; i < count; ++i) {
        const float* s = a.workspace + (REVERSE ? a.p.segments - 1 - i : i) * 2 * each;
        float m[C], v[C];
        load_floats<C>(m, s, at, p.channels);
        load_floats<C>(v, s + each, at, p.channels);
#pragma unroll
        for (int k = 0; k < C; ++k) h[k] = behind(m[k], v[k], h[k]);
    }
}

// Products and end values of each wave's part of a tile, [waves][64 * C] of them.
template <int C, int N>
struct Shared {
    float v[2][kMostWaves][N][kWave * C];
};

// Channels a lane takes, and the plan with it.
int channels_of(const ea_recurrence_t& c, bool backward);
Plan plan_of(const ea_recurrence_t& c, int channels);
constexpr int64_t kMostUnits = 1 << 20;                // workgroups of a launch; more work goes round

}  // namespace rec
}  // namespace ea
