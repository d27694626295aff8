// ea_adamw.hip -- AdamW over many tensors in one launch, with states in
// binary32 or in blockwise-scaled E4M3, and the global gradient norm.
//
// Both walk a table of tensors (parts of very large ones) that rides in the kernel's arguments: workgroup
// b belongs to the part whose range of workgroups holds b, found by one
// vector compare of the ranges' starts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_device.hpp"
#include "ea_train.hpp"

namespace ea {

namespace {

constexpr float kCodeMax = 448.0f;        // largest E4M3 value
constexpr float kLeastNormal = 0x1p-126f;

// b^t by square-and-multiply from the lowest bit.
__device__ __forceinline__ double ipow(double b, uint32_t t)
{
    double r = 1.0;
    for (; t; t >>= 1) {
        if (t & 1) r = r * b;
        b = b * b;
    }
    return r;
}

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

// The step's factors, formed once per workgroup.
struct Factors {
    float b1, a1, b2, a2, eps;
    float root;        // 1 / sqrt(1 - beta2^t)
    float step;        // lr_i / (1 - beta1^t)
    float keep;        // 1 - lr_i wd
    float gs;          // factor on the gradient
    uint32_t t;
};

__device__ __forceinline__ Factors factors_of(const AdamwArgs& a, const TensorPart& e, float gs)
{
    float lr = a.lr, beta2 = a.beta2;
    uint32_t t = a.t;
    if (a.t_dev) {
        t = *a.t_dev;
        schedule_at(a.sched, t, lr, beta2);
    }
    const double lri = (double)lr * (double)e.lr_scale;
    Factors f;
    f.t = t;
    f.gs = gs;
    f.b1 = a.beta1;
    f.a1 = (float)(1.0 - (double)a.beta1);
    f.b2 = beta2;
    f.a2 = (float)(1.0 - (double)beta2);
    f.eps = a.eps;
    f.root = (float)(1.0 / sqrt(1.0 - ipow((double)beta2, t)));
    f.step = (float)(lri / (1.0 - ipow((double)a.beta1, t)));
    f.keep = (float)(1.0 - lri * (double)e.weight_decay);
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

template <class P, class G>
__device__ __forceinline__ void adamw32_quad(const Factors& f, const TensorPart& e, int64_t i, int n)
{
    const G* gp = (const G*)e.g + i;
    P* pp = (P*)e.p + i;
    float* mp = (float*)e.m + i;
    float* vp = (float*)e.v + i;
    float* wp = e.master ? e.master + i : nullptr;
    const bool whole = n >= 4;
    const v4f g = widen(whole ? load4(gp) : load_some(gp, n));
    v4f m = whole ? load4(mp) : load_some(mp, n);
    v4f v = whole ? load4(vp) : load_some(vp, n);
    v4f p;
    if (wp)
        p = whole ? load4(wp) : load_some(wp, n);
    else
        p = widen(whole ? load4(pp) : load_some(pp, n));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float mk = m[k], vk = v[k], pk = p[k], r;
        adamw_element(f, g[k], mk, vk, r, pk);
        m[k] = mk;
        v[k] = vk;
        p[k] = pk;
    }
    if (whole) {
        store4(mp, m);
        store4(vp, v);
        if (wp) store4(wp, p);
        store4(pp, narrow<P>(p));
    } else {
        store_some(mp, m, n);
        store_some(vp, v, n);
        if (wp) store_some(wp, p, n);
        store_some(pp, narrow<P>(p), n);
    }
}

template <class P, class G>
__global__ void __launch_bounds__(kAdamwBlock) adamw32_kernel(AdamwArgs a)
{
    const float gs = a.gscale ? *a.gscale : 1.0f;
    if (!__builtin_isfinite(gs)) return;
    const int at = __builtin_amdgcn_readfirstlane(part_of<kListParts>(a.first, a.count, blockIdx.x));
    const TensorPart& e = a.part[at];
    const Factors f = factors_of(a, e, gs);
    const int64_t i = (int64_t)(blockIdx.x - a.first[at]) * (kAdamwBlock * 4) + threadIdx.x * 4;
    if (i < e.n) adamw32_quad<P, G>(f, e, i, e.n - i < 4 ? (int)(e.n - i) : 4);
}

// ---- states in 8 bits ------------------------------------------------------------

// Largest bit pattern of the wave: the largest magnitude of patterns without
// sign, an infinity above every number and a NaN above that.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v)
{
    v = max(v, dpp<kDppXor1>(v));
    v = max(v, dpp<kDppXor2>(v));
    v = max(v, dpp<kDppHalfMirror>(v));
    v = max(v, dpp<kDppRowMirror>(v));
    uint32_t a, b;
    row_swap16(v, a, b);
    v = max(a, b);
    row_swap32(v, a, b);
    return max(a, b);
}

__device__ __forceinline__ uint32_t magnitude(float x)
{
    return __float_as_uint(x) & 0x7FFFFFFFu;
}

// The block's scale from its largest magnitude: 0 below the normal numbers
// (the block is kept as zeros), NaN for an infinity or NaN (as is every value then).
__device__ __forceinline__ float block_scale(uint32_t top)
{
    const float s = __uint_as_float(top) * (1.0f / kCodeMax);
    if (top >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    return s < kLeastNormal ? 0.0f : s;
}

// |y| rounded by the 16-bit draw u to one of its two neighbours in E4M3, whose
// quantum is 2^-9 below 2^-6 and three fraction bits above.
__device__ __forceinline__ float round_by(float y, uint32_t u)
{
    const uint32_t up = (__float_as_uint(y) + ((u << 4) | 8u)) & ~0xFFFFFu;
    const float low = floorf(y * 512.0f + ((float)u + 0.5f) * 0x1p-16f) * 0x1p-9f;
    return y < 0x1p-6f ? low : __uint_as_float(up);
}

// Four values over the scale as E4M3 codes, one a byte.
template <bool DRAWS>
__device__ __forceinline__ uint32_t codes_of(v4f x, float scale, const uint32_t* u)
{
    if (!(scale > 0.0f)) return 0;
    const float inv = 1.0f / scale;
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a = fabsf(x[k] * inv);
        if (DRAWS) a = round_by(a, u[k]);
        y[k] = __builtin_copysignf(fminf(a, kCodeMax), x[k]);
    }
    uint32_t c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
}

__device__ __forceinline__ v4f values_of(uint32_t c, float scale)
{
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    return v4f{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
}

// A positive root's code 0 becomes 1 (2^-9 of the scale).
__device__ __forceinline__ uint32_t lift_zeros(uint32_t c, v4f r, float scale)
{
    if (!(scale > 0.0f)) return c;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (r[k] > 0.0f && ((c >> (8 * k)) & 0x7Fu) == 0) c |= 1u << (8 * k);
    return c;
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n)
{
    typedef uint32_t word __attribute__((aligned(1)));
    if (n >= 4) return *(const word*)p;
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
        *(word*)p = c;
        return;
    }
    if (n > 0) p[0] = (uint8_t)c;
    if (n > 1) p[1] = (uint8_t)(c >> 8);
    if (n > 2) p[2] = (uint8_t)(c >> 16);
}

// One wave, one block of 256 elements; lane l holds elements 4l to 4l+3.
template <class P, class G, bool DRAWS>
__global__ void __launch_bounds__(kAdamwBlock) adamw8_kernel(AdamwArgs a)
{
    const float gs = a.gscale ? *a.gscale : 1.0f;
    if (!__builtin_isfinite(gs)) return;
    const int at = __builtin_amdgcn_readfirstlane(part_of<kListParts>(a.first, a.count, blockIdx.x));
    const TensorPart& e = a.part[at];
    const Factors f = factors_of(a, e, gs);
    const int64_t block = (int64_t)(blockIdx.x - a.first[at]) * kWavesPerBlock + threadIdx.x / kWave;
    const int64_t i = block * EA_STATE_BLOCK + lane_id() * 4;
    if (block * EA_STATE_BLOCK >= e.n) return;
    const int n = i >= e.n ? 0 : e.n - i < 4 ? (int)(e.n - i) : 4;
    const bool whole = n == 4;
    const G* gp = (const G*)e.g + i;
    P* pp = (P*)e.p + i;
    uint8_t* mp = (uint8_t*)e.m + i;
    uint8_t* vp = (uint8_t*)e.v + i;
    float* wp = e.master ? e.master + i : nullptr;
    const v4f g = widen(whole ? load4(gp) : load_some(gp, n));
    v4f m = values_of(load_codes(mp, n), e.m_scale[block]);
    v4f r = values_of(load_codes(vp, n), e.v_scale[block]);
    v4f p;
    if (wp)
        p = whole ? load4(wp) : load_some(wp, n);
    else
        p = widen(whole ? load4(pp) : load_some(pp, n));
    uint32_t mtop = 0, rtop = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float mk = m[k], vk = r[k] * r[k], rk, pk = p[k];
        adamw_element(f, g[k], mk, vk, rk, pk);
        m[k] = mk;
        r[k] = rk;
        p[k] = pk;
        if (k < n) {
            mtop = max(mtop, magnitude(mk));
            rtop = max(rtop, magnitude(rk));
        }
    }
    const float ms = block_scale(wave_umax(mtop)), rs = block_scale(wave_umax(rtop));
    uint32_t um[4] = {0, 0, 0, 0}, ur[4] = {0, 0, 0, 0};
    if (DRAWS) {
        const uint64_t quad = ((uint64_t)e.piece * kPartElements + (uint64_t)i) >> 2;
        const uint4 w = philox10(make_uint4((uint32_t)quad, (uint32_t)(quad >> 32), f.t, e.index), a.k0, a.k1);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            um[k] = x[k] >> 16;
            ur[k] = x[k] & 0xFFFFu;
        }
    }
    const uint32_t cm = codes_of<DRAWS>(m, ms, um);
    const uint32_t cv = lift_zeros(codes_of<DRAWS>(r, rs, ur), r, rs);
    store_codes(mp, cm, n);
    store_codes(vp, cv, n);
    if (whole) {
        if (wp) store4(wp, p);
        store4(pp, narrow<P>(p));
    } else {
        if (wp) store_some(wp, p, n);
        store_some(pp, narrow<P>(p), n);
    }
    if (lane_id() == 0) {
        e.m_scale[block] = ms;
        e.v_scale[block] = rs;
    }
}

template <class P, class G>
void start_adamw(const AdamwArgs& a, const ea_adamw_t& c, hipStream_t s)
{
    const dim3 grid(a.first[a.count]), block(kAdamwBlock);
    if (c.state_bits == 32)
        hipLaunchKernelGGL((adamw32_kernel<P, G>), grid, block, 0, s, a);
    else if (c.rounding == EA_ROUND_STOCHASTIC)
        hipLaunchKernelGGL((adamw8_kernel<P, G, true>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((adamw8_kernel<P, G, false>), grid, block, 0, s, a);
}

template <class P>
void start_adamw_g(const AdamwArgs& a, const ea_adamw_t& c, hipStream_t s)
{
    if (c.grad_type == EA_F32)
        start_adamw<P, float>(a, c, s);
    else if (c.grad_type == EA_BF16)
        start_adamw<P, bf16>(a, c, s);
    else
        start_adamw<P, f16>(a, c, s);
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

template <class G>
__global__ void __launch_bounds__(kNormBlock) norm_kernel(NormArgs a)
{
    const int at = __builtin_amdgcn_readfirstlane(part_of<kNormParts>(a.first, a.count, blockIdx.x));
    const int64_t begin = (int64_t)(blockIdx.x - a.first[at]) * a.chunk;
    const int64_t n = a.part[at].n, end = begin + a.chunk < n ? begin + a.chunk : n;
    const G* g = (const G*)a.part[at].g;
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x * 4; i < end; i += kNormBlock * 4) {
        const v4f x = widen(end - i >= 4 ? load4(g + i) : load_some(g + i, (int)(end - i)));
#pragma unroll
        for (int k = 0; k < 4; ++k) sum = fma((double)x[k], (double)x[k], sum);
    }
    sum = block_sum<kNormBlock / kWave>(sum);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = sum;
}

constexpr int kFinishBlock = 1024;

__global__ void __launch_bounds__(kFinishBlock) norm_finish_kernel(const double* part, int64_t parts, float scale,
                                                                   float max_norm, float* norm, float* gscale)
{
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < parts; i += kFinishBlock) sum = sum + part[i];
    sum = block_sum<kFinishBlock / kWave>(sum);
    if (threadIdx.x == 0) {
        const float n = (float)((double)scale * sqrt(sum));
        float f = scale;
        if (!__builtin_isfinite(n))
            f = __uint_as_float(0x7FC00000u);
        else if (max_norm < n)
            f = (float)((double)scale * ((double)max_norm / (double)n));
        *norm = n;
        if (gscale) *gscale = f;
    }
}

}  // namespace

int64_t adamw_chunk(int64_t)
{
    return kAdamwBlock * 4;
}

hipError_t launch_adamw(const AdamwArgs& a, const ea_adamw_t& c, int64_t, hipStream_t s)
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

int64_t norm_chunk(int64_t total)
{
    int64_t c = 4096;
    while (total / c > 4096) c *= 2;
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

hipError_t launch_norm_finish(const double* part, int64_t parts, float scale, float max_norm, float* norm,
                              float* gscale, hipStream_t s)
{
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kFinishBlock), 0, s, part, parts, scale, max_norm, norm,
                       gscale);
    return hipGetLastError();
}

}  // namespace ea
