// ea_recurrence.hpp -- what the gated linear recurrence and its gradient share:
// the plan of a call, gates, loads of a wave's steps, and the states that
// chunks of a sequence hand on to each other.
//
// A workgroup takes a chunk of steps of 64 channels of one sequence, a channel a
// lane, so that every array passes memory once.  Each of its waves reads a few
// consecutive steps and runs them from a state of 0; the product of their gates
// and the state they end with go to LDS, and every wave folds what lies before
// it, in order, and runs its steps again from the true state.
//
// What a chunk starts with comes from the chunks before it through memory, by decoupled
// look-back (Merrill and Garland, 2016) with a fixed order of the fold.
// kGroup chunks form a group and kGroup groups a stretch.  A chunk hands out its
// product and end state as soon as it has them, without waiting for anything; the
// last chunk of a group folds the group's and hands that out; the last chunk of a
// stretch hands out the true state behind it.  So a chunk takes the state before
// its stretch and folds the groups, then the chunks before it, always in this
// order: the result does not depend on who came first, and only from stretch to
// stretch (65,536 steps forward) does one wait pass on to the next.
// Workgroups draw their chunks from a counter, in the order of the steps: who
// waits, waits for workgroups that have begun.  A wait of a good part of a second
// is given up, and the state is NaN.
//
// Bound by bytes and by what the exchange costs on top of them.  One sequence of
// 65,536 steps of 1,024 bfloat16 channels, states saved: 124 us, 3.3 TB/s; the
// gradient of 32 padded sequences of 2,048 steps (gates in binary32) 160 us, 4.5 TB/s;
// that of 2 x 16,384 x 768 binary32 with plain gates 117 us, 4.3 TB/s.  A lane is a
// channel, so that under 64 channels lanes idle and a row is one short load: what
// bounds is the steps, not the bytes (256 x 3,000 x 16 bfloat16 69 us, 1.1 TB/s;
// 64 x 8,000 x 32 57, 1.7; x 64 63, 3.1; the gradients 124, 96 and 105).  Other ways,
// before the results went past the caches (128 / 170 / 122 us then): steps as segments
// of whole sequences, the ends of which a first pass forms: 220 / 190 / 171.  Groups
// alone, without stretches: 124 / 168 / 122, but a wait that passes on every 4,096
// steps.  Three chunks in registers and one workgroup a CU, to have loads on
// their way during the exchange: 140 / 214 / 115; a wave of its own for the exchange:
// 207 / 333 / 160.
#pragma once

#include <type_traits>

#include "ea_layer.hpp"

namespace ea {
namespace rec {

constexpr int kMostWaves = 16;
constexpr int kGroup = 16;                             // chunks; a wave waits for each of those before
static_assert(kGroup <= kMostWaves, "a group's earlier chunks, and a stretch's earlier groups, have a wave each");

// Division of numbers under 2^31 by a number known to the host (Granlund and Montgomery, 1994): (h + (n - h) / 2) / 2^shift
// for the high half h of n * factor, in scalar instructions.
struct Divisor {
    uint32_t factor, shift, by;
    explicit Divisor(uint32_t d = 1) : by(d)
    {
        uint32_t bits = 0;
        while (((uint64_t)1 << bits) < d) ++bits;
        factor = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << bits) - d)) / d + 1);
        shift = bits;
    }
    __device__ uint32_t of(uint32_t n) const
    {
        const uint32_t h = __umulhi(factor, n);
        return shift == 0 ? n : (h + ((n - h) >> 1)) >> (shift - 1);
    }
};

struct Plan {
    uint32_t strips;                                   // of 64 channels
    uint32_t chunks, groups;                           // of a sequence
    int waves;                                         // of a chunk
};

// 64-bit words in the workspace: a counter, then for each chunk, sequence and channel the product and the end state,
// then the same for each group, then for each stretch the state before it.  The upper half of a word that has been
// handed out is 1: it and the value in the lower half become visible together, and nothing else has to be ordered.
struct Call {
    ea_recurrence_t c;
    Plan p;
    const int32_t* lengths;
    uint64_t* words;
    uint32_t items;                                    // strips * batch * chunks
    Divisor strips, batch, chunk;                      // chunk: its steps
};
constexpr int64_t kCounterWords = 16;

// The lane's place: sequence, chunk, channel.
struct Place {
    uint32_t b, chunk, channel;
    bool on;                                           // the lane has a channel
    int n;                                             // steps of the sequence that count
    uint32_t last;                                     // the chunk that has the last of them (0 when there is none)
};

__device__ __forceinline__ Place place_of(const Call& a, uint32_t item, bool reverse)
{
    Place p;
    const uint32_t rest = a.strips.of(item), strip = item - rest * a.p.strips;
    p.chunk = a.batch.of(rest);
    p.b = rest - p.chunk * (uint32_t)a.c.batch;
    if (reverse) p.chunk = a.p.chunks - 1 - p.chunk;
    p.channel = strip * kWave + lane_id();
    p.on = p.channel < (uint32_t)a.c.dim;
    p.n = (int)a.c.length;
    if (a.lengths) {
        const int n = uniform(a.lengths[p.b]);
        p.n = n < 0 ? 0 : n < p.n ? n : p.n;
    }
    p.last = p.n > 0 ? a.chunk.of((uint32_t)p.n - 1) : 0;
    return p;
}

// The workgroup's pieces of work, in turn.  With chains they are drawn from the counter, each while the one before is
// worked on: a piece that is drawn and not begun stands behind one that needs nothing from it.
template <bool CHAIN>
struct Items {
    uint32_t item;
    uint32_t* lds;
    __device__ void draw(const Call& a)
    {
        if (CHAIN && threadIdx.x == 0)
            *lds = (uint32_t)__hip_atomic_fetch_add((uint32_t*)a.words, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __device__ Items(const Call& a, uint32_t* at) : item(blockIdx.x), lds(at)
    {
        if (!CHAIN) return;
        draw(a);
        __syncthreads();
        item = (uint32_t)uniform((int)*lds);
        __syncthreads();
    }
    // behind a barrier after draw()
    __device__ void next(const Call& a)
    {
        item = CHAIN ? (uint32_t)uniform((int)*lds) : item + gridDim.x;
    }
};

// Words of the lane's channel: two of chunk `at` of all, or of group at - chunks; one of stretch `at`.
__device__ __forceinline__ uint64_t* pair_of(const Call& a, const Place& p, uint32_t at)
{
    return a.words + kCounterWords + (((int64_t)at * a.c.batch + p.b) * a.c.dim + p.channel) * 2;
}

__device__ __forceinline__ uint64_t* stretch_word(const Call& a, const Place& p, uint32_t stretch)
{
    const int64_t pairs = (int64_t)a.p.chunks + a.p.groups;
    return a.words + kCounterWords + ((pairs * 2 + stretch) * a.c.batch + p.b) * a.c.dim + p.channel;
}

__device__ __forceinline__ void hand_out(uint64_t* word, float v)
{
    __hip_atomic_store(word, (uint64_t)1 << 32 | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

constexpr int kMostPolls = 1 << 18;                    // about a microsecond each

// N consecutive words, once all have been handed out.
template <int N>
struct Wanted {
    uint64_t w[N];
    __device__ void ask(const uint64_t* from, bool on)
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            w[k] = on ? __hip_atomic_load(from + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : (uint64_t)1 << 32;
    }
    __device__ bool ready() const
    {
        bool all = true;
#pragma unroll
        for (int k = 0; k < N; ++k) all = all && w[k] >> 32 == 1;
        return all;
    }
    __device__ void wait(const uint64_t* from, bool on)
    {
        for (int i = 0; __ballot(!ready()) != 0; ++i) {
            if (i == kMostPolls) {
#pragma unroll
                for (int k = 0; k < N; ++k) w[k] = 0x7FC00000u;
                break;
            }
            __builtin_amdgcn_s_sleep(1);
            ask(from, on);
        }
    }
    __device__ float value(int k) const { return __uint_as_float((uint32_t)w[k]); }
};

// A row through a descriptor of its `dim` elements, or of none: lanes without a channel, and steps that do not count,
// read 0 and write nothing, and neither branches nor addresses take vector registers, so that 64 of them are enough and
// two workgroups share a CU.
template <class T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_of(const T* row, const Call& a, bool on)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)const_cast<T*>(row), 0, on ? (int)(a.c.dim * sizeof(T)) : 0,
                                             kRawBuffer);
}

template <class T>
__device__ __forceinline__ T load_own(__amdgpu_buffer_rsrc_t row, const Place& at)
{
    const uint32_t off = at.channel * (uint32_t)sizeof(T);
    if constexpr (sizeof(T) == 2)
        return __builtin_bit_cast(T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(row, off, 0, 0));
    else
        return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(row, off, 0, 0));
}

constexpr int kPastCaches = 2;                         // of a buffer store

template <int HOW, class T>
__device__ __forceinline__ void store_how(__amdgpu_buffer_rsrc_t row, uint32_t off, T v)
{
    if constexpr (sizeof(T) == 2)
        __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), row, off, 0, HOW);
    else
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), row, off, 0, HOW);
}

template <bool ONCE = false, class T>
__device__ __forceinline__ void store_own(__amdgpu_buffer_rsrc_t row, const Place& at, T v)
{
    store_how<ONCE ? kPastCaches : 0>(row, at.channel * (uint32_t)sizeof(T), v);
}

// A wave's steps from row `row` on, as they are stored; from step `count` on they are 0.
template <int K, class T>
__device__ __forceinline__ void load_steps(T* v, const T* p, int64_t row, int64_t stride, const Call& a,
                                           const Place& at, int count)
{
    const T* from = p + row * stride;
    if (count == K) {
#pragma unroll
        for (int k = 0; k < K; ++k, from += stride) v[k] = load_own<T>(row_of(from, a, true), at);
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k, from += stride) v[k] = load_own<T>(row_of(from, a, k < count), at);
}

// Steps that do not count keep the state.
template <int K>
__device__ __forceinline__ void mask_steps(float* f, float* v, int count)
{
    if (count == K) return;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        f[k] = k < count ? f[k] : 1.0f;
        v[k] = k < count ? v[k] : 0.0f;
    }
}

// Steps of the wave at step `t` before `end`, 0 to K.
template <int K>
__device__ __forceinline__ int steps_at(int64_t t, int end)
{
    const int64_t left = end - t;
    return left >= K ? K : left > 0 ? (int)left : 0;
}

// Zeros in the wave's steps that a sequence has no use for.
template <bool ONCE, class T>
__device__ __forceinline__ void zero_steps(T* p, int64_t row, int64_t stride, const Call& a, const Place& at, int from,
                                           int to)
{
    for (int k = from; k < to; ++k) store_own<ONCE>(row_of(p + (row + k) * stride, a, true), at, (T)0.0f);
}

// a and w of a gate: e / (1 + e) with e = exp(-|g|) for the smaller of them, and what is left of 1 for the other.  The
// larger is off by less than a rounding of its own where it is near 1: gates are multiplied over hundreds of steps.
template <bool SIGMOID>
__device__ __forceinline__ void gate_of(float g, float& a, float& w)
{
    if (!SIGMOID) {
        a = g;
        w = 1.0f;
        return;
    }
    const float e = __builtin_amdgcn_exp2f(-fabsf(g) * 0x1.715476p+0f);
    const float q = __builtin_amdgcn_rcpf(1.0f + e);
    const float s = e * q, r = __builtin_fmaf(-e, q, 1.0f);
    a = g < 0.0f ? s : r;
    w = g < 0.0f ? r : s;
}

// h behind steps whose gates' product is a and that lead from 0 to v.  A state of 0 stays out of the product: gates
// that multiply to infinity leave it what the steps one by one would.
__device__ __forceinline__ float behind(float a, float v, float h)
{
    return h == 0.0f ? v : __builtin_fmaf(a, h, v);
}

// One lane's value of a [batch, dim] array, 0 where there is none.
__device__ __forceinline__ float end_at(const float* p, const Call& a, const Place& at)
{
    return p && at.on ? p[at.b * a.c.dim + at.channel] : 0.0f;
}

struct Exchange {
    float wave[kMostWaves][3][kWave];                  // each wave's product, and what its steps lead to from 0
    float chunk[kGroup][2][kWave];                     // the same of the group's chunks before this one
    float group[kGroup][2][kWave];                     // of the stretch's groups before this one
    float start[kWave];                                // the state before the stretch
    uint32_t item;
};

// A chunk's place in its chain.
struct Link {
    int chunk, group;                                  // of its group, of its stretch
    uint32_t groups, stretch;                          // groups before its own, stretches before its own
    bool first, last;
};

__device__ __forceinline__ Link link_of(const Place& p, bool reverse)
{
    const uint32_t at = reverse ? p.last - p.chunk : p.chunk, groups = at / kGroup;
    return Link{(int)(at % kGroup), (int)(groups % kGroup), groups, groups / kGroup, at == 0, at == p.last};
}

// Hands out the chunk's product and end value (value `which` of each wave; REVERSE: from its last wave to its first)
// and gathers in LDS what fold_before() needs behind a barrier.
template <bool REVERSE>
__device__ __forceinline__ void meet(const Call& a, const Place& p, const Link& l, Exchange& x, int which,
                                     const float* start)
{
    const int wave = wave_id(), lane = lane_id();
    const bool ends = l.chunk == kGroup - 1 && !l.last;
    float m = 1.0f, v = 0.0f;
    if (wave == 0 && !l.last) {
#pragma unroll 4
        for (int i = 0; i < kMostWaves; ++i) {
            const int j = REVERSE ? kMostWaves - 1 - i : i;
            const float f = x.wave[j][0][lane];
            m = m * f;
            v = behind(f, x.wave[j][which][lane], v);
        }
        if (p.on && !ends) {
            uint64_t* to = pair_of(a, p, p.chunk);
            hand_out(to, m);
            hand_out(to + 1, v);
        }
    }
    // Each wave waits for one chunk, then one group; the last one for the state before the stretch.
    if (wave < l.chunk) {
        const int back = l.chunk - wave;               // chunks between that one and this
        const uint64_t* from = pair_of(a, p, REVERSE ? p.chunk + back : p.chunk - back);
        Wanted<2> chunk;
        chunk.ask(from, p.on);
        chunk.wait(from, p.on);
        x.chunk[wave][0][lane] = chunk.value(0);
        x.chunk[wave][1][lane] = chunk.value(1);
    }
    if (ends && l.group < kGroup - 1) {                // the group's, before anything else is waited for
        __syncthreads();
        if (wave == 0 && p.on) {
            float gm = 1.0f, gv = 0.0f;
#pragma unroll 4
            for (int i = 0; i < kGroup - 1; ++i) {
                gm = gm * x.chunk[i][0][lane];
                gv = behind(x.chunk[i][0][lane], x.chunk[i][1][lane], gv);
            }
            uint64_t* to = pair_of(a, p, a.p.chunks + l.groups);
            hand_out(to, gm * m);
            hand_out(to + 1, behind(m, v, gv));
        }
    }
    if (wave < l.group) {
        const uint64_t* from = pair_of(a, p, a.p.chunks + l.groups - l.group + wave);
        Wanted<2> group;
        group.ask(from, p.on);
        group.wait(from, p.on);
        x.group[wave][0][lane] = group.value(0);
        x.group[wave][1][lane] = group.value(1);
    }
    if (wave == kMostWaves - 1) {
        // The first chunk passes on what it starts with, too: the last one may write its own in the same place.
        if (l.first) {
            const float h = end_at(start, a, p);
            if (p.on && !l.last) hand_out(stretch_word(a, p, 0), h);
            x.start[lane] = h;
        } else {
            const uint64_t* from = stretch_word(a, p, l.stretch);
            Wanted<1> state;
            state.ask(from, p.on);
            state.wait(from, p.on);
            x.start[lane] = state.value(0);
        }
    }
}

// The state before the chunk.
__device__ __forceinline__ float fold_before(const Exchange& x, const Link& l)
{
    const int lane = lane_id();
    float h = x.start[lane];
#pragma unroll 4
    for (int i = 0; i < l.group; ++i) h = behind(x.group[i][0][lane], x.group[i][1][lane], h);
#pragma unroll 4
    for (int i = 0; i < l.chunk; ++i) h = behind(x.chunk[i][0][lane], x.chunk[i][1][lane], h);
    return h;
}

// Whether the true state behind the chunk is handed out.
__device__ __forceinline__ bool ends_stretch(const Link& l)
{
    return l.chunk == kGroup - 1 && l.group == kGroup - 1 && !l.last;
}

constexpr int kForwardSteps = 16, kBackwardSteps = 8;  // of a wave
Plan plan_of(const ea_recurrence_t& c, int steps);
int64_t words_of(const ea_recurrence_t& c, const Plan& p);
// The call, its words cleared; groups gets the workgroups of its launch, 0 for nothing to do.
hipError_t begin(Call& a, const ea_recurrence_t& c, int steps, const int32_t* lengths, void* workspace,
                 unsigned* groups, hipStream_t s);

// f with the types and the gate of a call as constants.
template <class F>
hipError_t with_kinds(const ea_recurrence_t& c, F&& f)
{
    return with_type(c.x_type, [&](auto x) {
        return with_type(c.g_type, [&](auto g) {
            return c.gate == EA_GATE_SIGMOID ? f(x, g, std::true_type{}) : f(x, g, std::false_type{});
        });
    });
}

}  // namespace rec
}  // namespace ea
