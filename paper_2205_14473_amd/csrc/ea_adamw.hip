// ea_adamw.hip -- AdamW over many tensors in one launch, with states in
// binary32 or in blockwise-scaled E4M3, and the global gradient norm.
//
// Both walk a table of tensors (parts of very large ones) that rides in the
// kernel's arguments: workgroup b belongs to the part whose range of workgroups
// holds b, found by one vector compare of the ranges' starts.  No table is
// uploaded and nothing is kept between calls; a list longer than the 4 KB of
// arguments takes further launches, whose starts and ends cost about 4 us each
// (355M parameters in 292 tensors: five with 32-bit states, 1% of the time, six
// with 8-bit ones, 4%).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_device.hpp"
#include "ea_train.hpp"

namespace ea {

namespace {

constexpr float kCodeMax = 448.0f;        // largest E4M3 value
constexpr float kLeastNormal = 0x1p-126f;

// lr and beta2 of the schedule at step t (as defined with ea_schedule_t).
__device__ __forceinline__ void schedule_at(const ea_schedule_t& s, uint32_t t, float& lr, float& beta2)
{
    if (s.kind == EA_SCHED_ASSUMPTION2) {
        const float Tf = (float)s.T;
        lr = s.alpha / sqrtf(Tf);
        beta2 = 1.0f - s.theta / Tf;
    } else if (s.kind == EA_SCHED_STEP_DECAY) {
        float r = 1.0f, b = s.factor;
        for (int64_t k = ((int64_t)t - 1) / s.period; k > 0; k >>= 1) {
            if (k & 1) r = r * b;
            b = b * b;
        }
        lr = s.alpha * r;
    }
}

// Index of the part that workgroup b works on: the last whose first
// workgroup is not after b.  Lane l compares entry l of the table.
template <int MOST>
__device__ __forceinline__ int part_of(const uint32_t* first, int count, uint32_t b)
{
    int at = -1;
    for (int k = 0; k < MOST; k += kWave) {
        const int l = k + lane_id();
        at += __popcll(__ballot(l < count && first[l] <= b));
    }
    return at;
}

// The step's factors, formed once per workgroup, before its loads where the step
// is read on the device: a scheduled step of 110M elements takes 1% longer with
// 32-bit states and 3 to 5% with 8-bit ones, of 65,536 elements 2.6 us longer
// (its launch that moves the step on among them).
struct Factors {
    float b1, a1, b2, a2, eps;
    float root;        // 1 / sqrt(1 - beta2^t)
    float step;        // lr_i / (1 - beta1^t)
    float keep;        // 1 - lr_i wd
    float gs;          // factor on the gradient
    uint32_t t;
};

template <class Args, class Part>
__device__ __forceinline__ Factors factors_of(const Args& a, const Part& e, float gs)
{
    Factors f;
    float lr = a.lr, beta2 = a.beta2;
    f.t = a.t;
    f.root = a.root;
    f.step = e.step;
    f.keep = e.keep;
    if (a.t_dev) {
        f.t = *a.t_dev;
        schedule_at(a.sched, f.t, lr, beta2);
        const double lri = (double)lr * (double)e.step;
        f.root = uniform(adamw_root(beta2, f.t));
        f.keep = uniform(adamw_keep(lri, e.keep));
        f.step = uniform(adamw_step_size(lri, a.beta1, f.t));
    }
    f.gs = gs;
    f.b1 = a.beta1;
    f.a1 = uniform(1.0f - a.beta1);      // the exact difference, rounded once
    f.b2 = beta2;
    f.a2 = uniform(1.0f - beta2);
    f.eps = a.eps;
    return f;
}

// One element: m, v and p in, m, v, its root and p out.
__device__ __forceinline__ void adamw_element(const Factors& f, float g, float& m, float& v, float& r, float& p)
{
    g = g * f.gs;
    m = m * f.b1 + g * f.a1;
    v = v * f.b2 + (g * g) * f.a2;
    r = sqrtf(v);
    p = p * f.keep - (m / (r * f.root + f.eps)) * f.step;
}

// ---- states in 32 bits ---------------------------------------------------------

constexpr int kAdamwBlock = 256;

// m, v and p of one quad:
//     m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g g;  p <- keep p - step m / (root sqrt(v) + eps)
// HBM bounds it: 28 bytes an element move once, and the arithmetic (45
// instructions, with root and quotient rounded as IEEE 754 has them) takes half
// of that time.  355M parameters (bfloat16 with binary32 masters) 1.65 ms, 6.0
// TB/s; 110M (binary32, bfloat16 gradients) 473 us, 6.0; 11.7M in 62 tensors off
// alignment 58 us, 5.6.  One quad a thread and many workgroups: with two or four
// quads a thread, their loads ahead of the arithmetic, the first took 1.69 and
// 1.71 ms.  Every byte is used once, so loads and stores pass the caches by
// (1.83 ms through them).
template <class P, class G>
__device__ __forceinline__ void adamw32_quad(const Factors& f, const Part32& e, uint32_t i, int n)
{
    const G* gp = (const G*)e.g + i;
    P* pp = (P*)e.p + i;
    float* mp = (float*)e.m + i;
    float* vp = (float*)e.v + i;
    float* wp = e.master ? e.master + i : nullptr;
    const bool four = n == 4;
    const v4f g = widen(four ? load4_once(gp) : load_some(gp, n));
    v4f m = four ? load4_once(mp) : load_some(mp, n);
    v4f v = four ? load4_once(vp) : load_some(vp, n);
    v4f p;
    if (wp)
        p = four ? load4_once(wp) : load_some(wp, n);
    else
        p = widen(four ? load4_once(pp) : load_some(pp, n));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float mk = m[k], vk = v[k], pk = p[k], r;
        adamw_element(f, g[k], mk, vk, r, pk);
        m[k] = mk;
        v[k] = vk;
        p[k] = pk;
    }
    if (four) {
        store4_once(mp, m);
        store4_once(vp, v);
        if (wp) store4_once(wp, p);
        store4_once(pp, narrow<P>(p));
    } else {
        store_some(mp, m, n);
        store_some(vp, v, n);
        if (wp) store_some(wp, p, n);
        store_some(pp, narrow<P>(p), n);
    }
}

template <class P, class G>
__global__ void __launch_bounds__(kAdamwBlock) adamw32_kernel(Adamw32Args a)
{
    const float gs = a.gscale ? *a.gscale : 1.0f;
    if (!__builtin_isfinite(gs)) return;
    const int at = __builtin_amdgcn_readfirstlane(part_of<Adamw32Args::kMost>(a.first, a.count, blockIdx.x));
    const Part32& e = a.part[at];
    const Factors f = factors_of(a, e, gs);
    const uint32_t i = ((blockIdx.x - a.first[at]) * kAdamwBlock + threadIdx.x) * 4;
    if (i < e.n) adamw32_quad<P, G>(f, e, i, e.n - i < 4 ? (int)(e.n - i) : 4);
}

// ---- states in 8 bits ------------------------------------------------------------

constexpr int kRowLanes = 32;            // lanes that share a block of the 8-bit states

// Largest bit pattern of a half wave: of patterns without sign, an infinity
// stands above every number and a NaN above that.
__device__ __forceinline__ uint32_t row_umax(uint32_t v)
{
    v = max(v, dpp<kDppXor1>(v));
    v = max(v, dpp<kDppXor2>(v));
    v = max(v, dpp<kDppHalfMirror>(v));
    v = max(v, dpp<kDppRowMirror>(v));
    uint32_t a, b;
    row_swap16(v, a, b);
    return max(a, b);
}

__device__ __forceinline__ uint32_t magnitude(float x)
{
    return __float_as_uint(x) & 0x7FFFFFFFu;
}

// The block's scale from its largest magnitude: 0 below the normal numbers
// (the block is kept as zeros), NaN for an infinity or NaN (as is every value
// then).  `inv` is 1 / scale, and 0 in both those cases.
__device__ __forceinline__ float block_scale(uint32_t top, float& inv)
{
    float s = __uint_as_float(top) * (1.0f / kCodeMax);
    s = s < kLeastNormal ? 0.0f : s;
    const bool odd = top >= 0x7F800000u;
    inv = s > 0.0f && !odd ? 1.0f / s : 0.0f;
    return odd ? __uint_as_float(0x7FC00000u) : s;
}

// y >= 0 rounded by the 16-bit draw u to one of its two neighbours in E4M3, whose
// quantum is 2^-9 below 2^-6 and three fraction bits above.
__device__ __forceinline__ float round_by(float y, uint32_t u)
{
    const uint32_t up = (__float_as_uint(y) + ((u << 4) | 8u)) & ~0xFFFFFu;
    const float low = floorf(fmaf(y, 512.0f, fmaf((float)u, 0x1p-16f, 0x1p-17f))) * 0x1p-9f;   // products are exact
    return fminf(y < 0x1p-6f ? low : __uint_as_float(up), kCodeMax);
}

// A value over its block's scale, on or between E4M3 numbers: with a finite
// value at most 448 and a few units in the last place, which the conversion
// rounds to 448.  (With inv = 0 an infinity or NaN becomes a NaN: the scale says so.)
template <bool DRAWS>
__device__ __forceinline__ float over_scale(float x, float inv, uint32_t u)
{
    const float y = x * inv;
    return DRAWS ? __builtin_copysignf(round_by(fabsf(y), u), y) : y;
}

// The same of a root.  A positive one is at least `least`, 2^-9 (0 where inv
// is 0): below it, to nearest, are 0 and that code only.
template <bool DRAWS>
__device__ __forceinline__ float root_over_scale(float x, float inv, float least, uint32_t u)
{
    const float y = fmaxf(x * inv, x > 0.0f ? least : 0.0f);
    return DRAWS ? round_by(y, u) : y;
}

__device__ __forceinline__ uint32_t pack_codes(const float* y)
{
    const uint32_t c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
}

__device__ __forceinline__ v4f values_of(uint32_t c, float scale)
{
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    return v4f{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n)
{
    typedef uint32_t word __attribute__((aligned(1)));
    if (n >= 4) return __builtin_nontemporal_load((const word*)p);
    uint32_t c = 0;
    if (n > 0) c |= p[0];
    if (n > 1) c |= (uint32_t)p[1] << 8;
    if (n > 2) c |= (uint32_t)p[2] << 16;
    return c;
}

__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t c, int n)
{
    typedef uint32_t word __attribute__((aligned(1)));
    if (n >= 4) {
        __builtin_nontemporal_store(c, (word*)p);
        return;
    }
    if (n > 0) p[0] = (uint8_t)c;
    if (n > 1) p[1] = (uint8_t)(c >> 8);
    if (n > 2) p[2] = (uint8_t)(c >> 16);
}

constexpr int kRowQuads = EA_STATE_BLOCK / 4 / kRowLanes;
constexpr uint32_t kWaveElements = (kWave / kRowLanes) * EA_STATE_BLOCK;

// Root and quotient by one correction step on the hardware's approximations
// (each within one unit in the last place): what is left before the last
// rounding is of second order, some 2^-21 of a unit for the quotient's and the
// root's alike, so the result is one of the value's two neighbours, and for all
// but about one value in a million the nearer, as sqrtf and the division give.  Those two check for operands that
// the approximations do not take (29 instructions an element together, of 45;
// here 12), which is left to plain_square below.
__device__ __forceinline__ float root_of(float v)
{
    const float y = __builtin_amdgcn_rsqf(fmaxf(v, kLeastNormal));
    const float s = v * y;
    return fmaf(fmaf(-s, s, v), 0.5f * y, s);
}

__device__ __forceinline__ float quotient(float a, float b)
{
    float y = __builtin_amdgcn_rcpf(b);
    y = fmaf(fmaf(-b, y, 1.0f), y, y);
    const float q = a * y;
    return fmaf(fmaf(-b, q, a), y, q);
}

// Neither subnormal, infinite nor NaN.
__device__ __forceinline__ bool plain_square(float v)
{
    return !__builtin_amdgcn_classf(v, 0x003 | 0x004 | 0x010 | 0x080 | 0x200);
}

// A wave takes one group of blocks; where parameters and gradients have 16 bits
// and no masters stand behind them, four from this many elements on (twice as
// many with draws), with the next one's loads in flight: with few bytes in
// flight a lane, waves that start and end leave HBM idle (both 16 bits, us for
// one and four a wave: 2^23 elements 29.6 and 32.4, 2^25 76.8 and 73.3, 2^27 278
// and 256; with draws 2^25 89.8 and 93.0, 2^26 170.6 and 167.3).  Others
// have enough in flight and lose by the longer runs and their registers: 2^27 of
// binary32 340 and 383, binary32 with bfloat16 gradients 303 and 333, bfloat16
// with masters 352 and 384, with binary32 gradients 269 and 288.
constexpr int64_t kLongRuns = 1 << 25;
constexpr float kLeastEps = 0x1p-100f;   // outside these two, quotient's reciprocal could leave the
constexpr float kMostEps = 0x1p100f;     // normal numbers
constexpr float kMostOverEps = 0x1p120f; // first moments over eps from which it could overflow (and end as
                                         // inf - inf where the division gives an infinity)

// The codes of a quad of first moments and roots, in place of the old ones.
template <bool DRAWS>
__device__ __forceinline__ void store_states(const Adamw8Args& a, const Factors& f, const Part8& e, uint32_t at,
                                             uint8_t* mp, uint8_t* vp, v4f m, v4f r, float minv, float rinv, int n)
{
    const float least = rinv > 0.0f ? 0x1p-9f : 0.0f;
    uint4 w = {0, 0, 0, 0};
    if (DRAWS) {
        const uint64_t quad = ((uint64_t)(e.place & ((1u << kPieceBits) - 1)) * kPartElements + at) >> 2;
        w = philox10(make_uint4((uint32_t)quad, (uint32_t)(quad >> 32), f.t, e.place >> kPieceBits), a.k0, a.k1);
    }
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    float ym[4], yr[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        ym[k] = over_scale<DRAWS>(m[k], minv, u[k] >> 16);
        yr[k] = root_over_scale<DRAWS>(r[k], rinv, least, u[k] & 0xFFFFu);
    }
    store_codes(mp, pack_codes(ym), n);
    store_codes(vp, pack_codes(yr), n);
}

// The step on blocks of 256 elements whose m and r = sqrt(v) are kept as E4M3
// codes under a scale each:
//     m = code scale, v = (code scale)^2;  the step as above;  r = sqrt(v)
//     scale <- max|x| / 448, code <- round(x / scale)
// A wave has two blocks, each on half of its lanes, a lane the block's quads j
// and j + 32: the largest magnitude takes five steps without LDS, loads stay
// side by side, and the scales' divisions serve eight elements a lane.  (With 16
// lanes a block, and 16 elements a lane, registers halve the waves: 771 us
// against 661 for 355M; with 64 the reduction and the divisions cost more, 739
// against 689 before loads went ahead.)
// 10 bytes an element (bfloat16 parameters and gradients) against 200
// instructions for 256 elements: vector issue is busy three quarters of the time
// beside HBM at 5.4 TB/s, 355M parameters 656 us.  With stochastic rounding the
// draws double the instructions: 11.7M 41 us, 4.6 TB/s (16 bytes an element).
//
// This is the form for any values and any number of elements.
template <class P, class G, bool DRAWS>
__device__ __forceinline__ void adamw8_any(const Adamw8Args& a, const Factors& f, const Part8& e, uint32_t begin)
{
    const int lane = lane_id(), row = lane / kRowLanes;
    const uint32_t block = begin / EA_STATE_BLOCK + row;
    if (block * (uint64_t)EA_STATE_BLOCK >= e.n) return;
    const float ms0 = e.m_scale[block], rs0 = e.v_scale[block];
    v4f m[kRowQuads], r[kRowQuads];
    uint32_t mtop = 0, rtop = 0;
#pragma unroll
    for (int q = 0; q < kRowQuads; ++q) {
        const uint32_t i = block * EA_STATE_BLOCK + (q * kRowLanes + lane % kRowLanes) * 4;
        const int n = i >= e.n ? 0 : e.n - i < 4 ? (int)(e.n - i) : 4;
        const G* gp = (const G*)e.g + i;
        P* pp = (P*)e.p + i;
        float* wp = e.master ? e.master + i : nullptr;
        const v4f g = widen(n == 4 ? load4_once(gp) : load_some(gp, n));
        v4f p;
        if (wp)
            p = n == 4 ? load4_once(wp) : load_some(wp, n);
        else
            p = widen(n == 4 ? load4_once(pp) : load_some(pp, n));
        m[q] = values_of(load_codes((uint8_t*)e.m + i, n), ms0);
        r[q] = values_of(load_codes((uint8_t*)e.v + i, n), rs0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float mk = m[q][k], vk = r[q][k] * r[q][k], rk, pk = p[k];
            adamw_element(f, g[k], mk, vk, rk, pk);
            m[q][k] = mk;
            r[q][k] = rk;
            p[k] = pk;
            if (k < n) {
                mtop = max(mtop, magnitude(mk));
                rtop = max(rtop, magnitude(rk));
            }
        }
        if (n == 4) {
            if (wp) store4_once(wp, p);
            store4_once(pp, narrow<P>(p));
        } else {
            if (wp) store_some(wp, p, n);
            store_some(pp, narrow<P>(p), n);
        }
    }
    float minv, rinv;
    const float ms = block_scale(row_umax(mtop), minv), rs = block_scale(row_umax(rtop), rinv);
#pragma unroll
    for (int q = 0; q < kRowQuads; ++q) {
        const uint32_t i = block * EA_STATE_BLOCK + (q * kRowLanes + lane % kRowLanes) * 4;
        const int n = i >= e.n ? 0 : e.n - i < 4 ? (int)(e.n - i) : 4;
        store_states<DRAWS>(a, f, e, i, (uint8_t*)e.m + i, (uint8_t*)e.v + i, m[q], r[q], minv, rinv, n);
    }
    if (lane % kRowLanes == 0) {
        e.m_scale[block] = ms;
        e.v_scale[block] = rs;
    }
}

// What a lane reads of its block, as it is kept.
template <class P, class G, bool MASTER>
struct Held {
    uint32_t cm[kRowQuads], cr[kRowQuads];
    typename Quad<G>::vec g[kRowQuads];
    typename Quad<P>::vec p[kRowQuads];
    v4f w[kRowQuads];
    float ms, rs;
};

// First of a lane's elements among its wave's; its others follow 4 kRowLanes apart.
__device__ __forceinline__ uint32_t first_of_lane()
{
    return (lane_id() / kRowLanes) * EA_STATE_BLOCK + (lane_id() % kRowLanes) * 4;
}

template <class P, class G, bool MASTER>
__device__ __forceinline__ void fetch(const Part8& e, uint32_t begin, Held<P, G, MASTER>& h)
{
    const int row = lane_id() / kRowLanes;
    h.ms = (e.m_scale + begin / EA_STATE_BLOCK)[row];
    h.rs = (e.v_scale + begin / EA_STATE_BLOCK)[row];
#pragma unroll
    for (int q = 0; q < kRowQuads; ++q) {
        const uint32_t at = first_of_lane() + q * kRowLanes * 4;
        h.cm[q] = load_codes((const uint8_t*)e.m + begin + at, 4);
        h.cr[q] = load_codes((const uint8_t*)e.v + begin + at, 4);
        h.g[q] = load4_once((const G*)e.g + begin + at);
        if (MASTER)
            h.w[q] = load4_once(e.master + begin + at);
        else
            h.p[q] = load4_once((const P*)e.p + begin + at);
    }
}

// The same for whole blocks, fetched before, and values that root_of and
// quotient take, as nearly all are; false, with nothing written, where one is not.
template <class P, class G, bool DRAWS, bool MASTER>
__device__ __forceinline__ bool adamw8_whole(const Adamw8Args& a, const Factors& f, const Part8& e, uint32_t begin,
                                             const Held<P, G, MASTER>& h)
{
    const uint32_t first = first_of_lane();
    v4f p[kRowQuads], m[kRowQuads], r[kRowQuads];
    float mtop = 0.0f, rtop = 0.0f;
    bool fine = true;
#pragma unroll
    for (int q = 0; q < kRowQuads; ++q) {
        m[q] = values_of(h.cm[q], h.ms);
        r[q] = values_of(h.cr[q], h.rs);
        p[q] = MASTER ? h.w[q] : widen(h.p[q]);
        const v4f g = widen(h.g[q]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gk = g[k] * f.gs;
            const float mk = m[q][k] * f.b1 + gk * f.a1;
            const float vk = (r[q][k] * r[q][k]) * f.b2 + (gk * gk) * f.a2;
            const float rk = root_of(vk);
            fine &= plain_square(vk);
            p[q][k] = p[q][k] * f.keep - quotient(mk, rk * f.root + f.eps) * f.step;
            m[q][k] = mk;
            r[q][k] = rk;
            mtop = __builtin_elementwise_maximum(mtop, fabsf(mk));  // a NaN stays
            rtop = fmaxf(rtop, rk);
        }
    }
    fine &= mtop < f.eps * kMostOverEps;                   // nor NaN
    if (__ballot(!fine)) return false;
#pragma unroll
    for (int q = 0; q < kRowQuads; ++q) {
        const uint32_t at = begin + first + q * kRowLanes * 4;
        if (MASTER) store4_once(e.master + at, p[q]);
        store4_once((P*)e.p + at, narrow<P>(p[q]));
    }
    float minv, rinv;
    const float ms = block_scale(row_umax(__float_as_uint(mtop)), minv);
    const float rs = block_scale(row_umax(__float_as_uint(rtop)), rinv);
#pragma unroll
    for (int q = 0; q < kRowQuads; ++q) {
        const uint32_t at = begin + first + q * kRowLanes * 4;
        store_states<DRAWS>(a, f, e, at, (uint8_t*)e.m + at, (uint8_t*)e.v + at, m[q], r[q], minv, rinv, 4);
    }
    if (lane_id() % kRowLanes == 0) {
        (e.m_scale + begin / EA_STATE_BLOCK)[lane_id() / kRowLanes] = ms;
        (e.v_scale + begin / EA_STATE_BLOCK)[lane_id() / kRowLanes] = rs;
    }
    return true;
}

// A wave's run of its part: whole groups of blocks, each fetched before the
// last one is worked on, then what is left of the part.
template <class P, class G, bool DRAWS, bool MASTER>
__device__ __forceinline__ void adamw8_run(const Adamw8Args& a, const Factors& f, const Part8& e, uint32_t begin,
                                           uint32_t end)
{
    constexpr bool kSeveral = sizeof(P) == 2 && sizeof(G) == 2 && !MASTER;   // adamw_chunk's runs of four
    Held<P, G, MASTER> h, next;
    if (f.eps >= kLeastEps && f.eps <= kMostEps && end - begin >= kWaveElements) {
        fetch<P, G, MASTER>(e, begin, h);
        for (;;) {
            const uint32_t then = begin + kWaveElements;
            const bool more = kSeveral && end - then >= kWaveElements;
            if (more) fetch<P, G, MASTER>(e, then, next);
            if (!adamw8_whole<P, G, DRAWS, MASTER>(a, f, e, begin, h)) adamw8_any<P, G, DRAWS>(a, f, e, begin);
            begin = then;
            if (!more) break;
            h = next;
        }
    }
    for (; begin < end; begin += kWaveElements) adamw8_any<P, G, DRAWS>(a, f, e, begin);
}

template <class P, class G, bool DRAWS>
__global__ void __launch_bounds__(kAdamwBlock) adamw8_kernel(Adamw8Args a)
{
    const float gs = a.gscale ? *a.gscale : 1.0f;
    if (!__builtin_isfinite(gs)) return;
    const int at = __builtin_amdgcn_readfirstlane(part_of<Adamw8Args::kMost>(a.first, a.count, blockIdx.x));
    const Part8& e = a.part[at];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), run = a.chunk / kWavesPerBlock;
    const uint32_t begin = ((blockIdx.x - a.first[at]) * kWavesPerBlock + wave) * run;
    if (begin >= e.n) return;
    const uint32_t end = e.n - begin < run ? e.n : begin + run;
    const Factors f = factors_of(a, e, gs);
    if (sizeof(P) == 2 && e.master)
        adamw8_run<P, G, DRAWS, true>(a, f, e, begin, end);
    else
        adamw8_run<P, G, DRAWS, false>(a, f, e, begin, end);
}

template <class P, class G>
void start_adamw(const Adamw32Args& a, const ea_adamw_t&, hipStream_t s)
{
    hipLaunchKernelGGL((adamw32_kernel<P, G>), dim3(a.first[a.count]), dim3(kAdamwBlock), 0, s, a);
}

template <class P, class G>
void start_adamw(const Adamw8Args& a, const ea_adamw_t& c, hipStream_t s)
{
    const dim3 grid(a.first[a.count]), block(kAdamwBlock);
    if (c.rounding == EA_ROUND_STOCHASTIC)
        hipLaunchKernelGGL((adamw8_kernel<P, G, true>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((adamw8_kernel<P, G, false>), grid, block, 0, s, a);
}

template <class P, class Args>
void start_adamw_g(const Args& a, const ea_adamw_t& c, hipStream_t s)
{
    if (c.grad_type == EA_F32)
        start_adamw<P, float>(a, c, s);
    else if (c.grad_type == EA_BF16)
        start_adamw<P, bf16>(a, c, s);
    else
        start_adamw<P, f16>(a, c, s);
}

template <class Args>
hipError_t start_adamw_p(const Args& a, const ea_adamw_t& c, hipStream_t s)
{
    if (a.count < 1 || a.first[a.count] == 0) return hipSuccess;
    if (c.param_type == EA_F32)
        start_adamw_g<float>(a, c, s);
    else if (c.param_type == EA_BF16)
        start_adamw_g<bf16>(a, c, s);
    else
        start_adamw_g<f16>(a, c, s);
    return hipGetLastError();
}

// ---- gradient norm -----------------------------------------------------------------

constexpr int kNormBlock = 256;

// Sum over a workgroup, the same bits on every run; valid on thread 0.
template <int WAVES>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[WAVES];
    v = wave_sum(v);
    if (lane_id() == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    double r = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < WAVES; ++w) r = r + part[w];
    return r;
}

// sum of g^2 in binary64: binary32 squares overflow above 1.8e19 and vanish under
// 1e-23, and the wider sum is free beside HBM.  Chunks' sums are joined by a
// second launch, in an order that the list alone fixes.  355M bfloat16 gradients
// 111 us, 6.4 TB/s, with 8192 chunks (4096: 124; loads through the caches: 138);
// 29.8M in 75 tensors 12.9 with 16,384 elements a chunk (8,192: 14.8, 4,096: 19.9).
//
// Squares of n elements summed over the workgroup's threads, in 16-byte loads,
// eight in flight a thread, then four, two and one.
template <class G, int THREADS>
__device__ __forceinline__ double squares(const G* g, uint32_t n)
{
    constexpr int kEach = 16 / sizeof(G);
    typedef G vec __attribute__((ext_vector_type(kEach)));
    typedef vec unaligned __attribute__((aligned(sizeof(G))));
    constexpr uint32_t kStride = THREADS * kEach;
    double sum = 0.0;
    const auto add = [&sum](float x) { sum = fma((double)x, (double)x, sum); };
    uint32_t i = threadIdx.x * kEach;
    const auto take = [&](auto ahead) {
        vec x[ahead.value];
#pragma unroll
        for (int u = 0; u < ahead.value; ++u) x[u] = __builtin_nontemporal_load((const unaligned*)(g + i + u * kStride));
#pragma unroll
        for (int u = 0; u < ahead.value; ++u)
#pragma unroll
            for (int k = 0; k < kEach; ++k) add((float)x[u][k]);
        i += ahead.value * kStride;
    };
    const auto fit = [&](int ahead) { return (uint64_t)i + (ahead - 1) * kStride + kEach <= n; };
    while (fit(8)) take(std::integral_constant<int, 8>());
    if (fit(4)) take(std::integral_constant<int, 4>());
    if (fit(2)) take(std::integral_constant<int, 2>());
    if (fit(1)) take(std::integral_constant<int, 1>());
    if (i < n)
        for (uint32_t k = 0; k < kEach && k < n - i; ++k) add((float)g[i + k]);
    return sum;
}

template <class G>
__global__ void __launch_bounds__(kNormBlock) norm_kernel(NormArgs a)
{
    const int at = __builtin_amdgcn_readfirstlane(part_of<kNormParts>(a.first, a.count, blockIdx.x));
    const int64_t begin = (int64_t)(blockIdx.x - a.first[at]) * a.chunk, left = a.part[at].n - begin;
    const uint32_t n = (uint32_t)(left < a.chunk ? left : a.chunk);
    const double sum =
        block_sum<kNormBlock / kWave>(squares<G, kNormBlock>((const G*)a.part[at].g + begin, n));
    if (threadIdx.x == 0) a.sums[blockIdx.x] = sum;
}

// Norm and factor from the sum of squares.
__device__ __forceinline__ void norm_out(double sum, float scale, float max_norm, float* norm, float* gscale)
{
    const float n = (float)((double)scale * sqrt(sum));
    float f = scale;
    if (!__builtin_isfinite(n))
        f = __uint_as_float(0x7FC00000u);
    else if (max_norm < n)
        f = (float)((double)scale * ((double)max_norm / (double)n));
    *norm = n;
    if (gscale) *gscale = f;
}

constexpr int kFinishBlock = 1024;

__global__ void __launch_bounds__(kFinishBlock) norm_finish_kernel(const double* part, int64_t parts, float scale,
                                                                   float max_norm, float* norm, float* gscale)
{
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < parts; i += kFinishBlock) sum = sum + part[i];
    sum = block_sum<kFinishBlock / kWave>(sum);
    if (threadIdx.x == 0) norm_out(sum, scale, max_norm, norm, gscale);
}

// Few elements: one launch of one workgroup.
template <class G>
__global__ void __launch_bounds__(kFinishBlock) norm_small_kernel(NormArgs a, float scale, float max_norm, float* norm,
                                                                  float* gscale)
{
    double sum = 0.0;
    for (int k = 0; k < a.count; ++k) sum = sum + squares<G, kFinishBlock>((const G*)a.part[k].g, (uint32_t)a.part[k].n);
    sum = block_sum<kFinishBlock / kWave>(sum);
    if (threadIdx.x == 0) norm_out(sum, scale, max_norm, norm, gscale);
}

}  // namespace

uint32_t adamw_chunk(const ea_adamw_t& c, int64_t total, bool masters)
{
    if (c.state_bits == 32) return kAdamwBlock * 4;
    const bool light = c.param_type != EA_F32 && c.grad_type != EA_F32 && !masters;
    const bool many = total >= (c.rounding == EA_ROUND_STOCHASTIC ? 2 * kLongRuns : kLongRuns);
    return kWavesPerBlock * kWaveElements * (light && many ? 4 : 1);
}

hipError_t launch_adamw(const Adamw32Args& a, const ea_adamw_t& c, hipStream_t s)
{
    return start_adamw_p(a, c, s);
}

hipError_t launch_adamw(const Adamw8Args& a, const ea_adamw_t& c, hipStream_t s)
{
    return start_adamw_p(a, c, s);
}

int64_t norm_chunk(int64_t total)
{
    int64_t c = 16384;
    while (total / c > 8192) c *= 2;
    return c;
}

hipError_t launch_norm(const NormArgs& a, int32_t grad_type, hipStream_t s)
{
    if (a.count < 1 || a.first[a.count] == 0) return hipSuccess;
    const dim3 grid(a.first[a.count]), block(kNormBlock);
    if (grad_type == EA_F32)
        hipLaunchKernelGGL(norm_kernel<float>, grid, block, 0, s, a);
    else if (grad_type == EA_BF16)
        hipLaunchKernelGGL(norm_kernel<bf16>, grid, block, 0, s, a);
    else
        hipLaunchKernelGGL(norm_kernel<f16>, grid, block, 0, s, a);
    return hipGetLastError();
}

bool norm_in_one(const NormArgs& a, int64_t total)
{
    return a.count <= kSmallParts && total <= kSmallTotal;
}

hipError_t launch_norm_small(const NormArgs& a, int32_t grad_type, float scale, float max_norm, float* norm,
                             float* gscale, hipStream_t s)
{
    const dim3 grid(1), block(kFinishBlock);
    if (grad_type == EA_F32)
        hipLaunchKernelGGL(norm_small_kernel<float>, grid, block, 0, s, a, scale, max_norm, norm, gscale);
    else if (grad_type == EA_BF16)
        hipLaunchKernelGGL(norm_small_kernel<bf16>, grid, block, 0, s, a, scale, max_norm, norm, gscale);
    else
        hipLaunchKernelGGL(norm_small_kernel<f16>, grid, block, 0, s, a, scale, max_norm, norm, gscale);
    return hipGetLastError();
}

hipError_t launch_norm_finish(const double* part, int64_t parts, float scale, float max_norm, float* norm,
                              float* gscale, hipStream_t s)
{
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kFinishBlock), 0, s, part, parts, scale, max_norm, norm,
                       gscale);
    return hipGetLastError();
}

}  // namespace ea
