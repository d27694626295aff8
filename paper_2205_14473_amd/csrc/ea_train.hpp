// ea_train.hpp -- argument blocks, element types and launchers of the
// operators beside the round (ea_train.h): AdamW over many tensors, gradient
// norm, embedding.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea_train.h"

namespace ea {

// ---- element types ----------------------------------------------------------

using bf16 = __bf16;
using f16 = _Float16;
using v4f = float __attribute__((ext_vector_type(4)));

// Four consecutive elements of type T at an address aligned to one element:
// gfx950 loads and stores vectors at any such address.
template <class T>
struct Quad {
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec unaligned __attribute__((aligned(sizeof(T))));
};

template <class T>
__device__ __forceinline__ typename Quad<T>::vec load4(const T* p)
{
    return *(const typename Quad<T>::unaligned*)p;
}

template <class T>
__device__ __forceinline__ void store4(T* p, typename Quad<T>::vec v)
{
    *(typename Quad<T>::unaligned*)p = v;
}

// The same for data that a pass reads or writes once: it leaves the caches to others.
template <class T>
__device__ __forceinline__ typename Quad<T>::vec load4_once(const T* p)
{
    return __builtin_nontemporal_load((const typename Quad<T>::unaligned*)p);
}

template <class T>
__device__ __forceinline__ void store4_once(T* p, typename Quad<T>::vec v)
{
    __builtin_nontemporal_store(v, (typename Quad<T>::unaligned*)p);
}

template <class T>
__device__ __forceinline__ v4f widen(T v)
{
    return __builtin_convertvector(v, v4f);
}

template <class T>
__device__ __forceinline__ typename Quad<T>::vec narrow(v4f v)
{
    return __builtin_convertvector(v, typename Quad<T>::vec);
}

// The first `n` (0 to 3) of four elements; the rest read as zeros, and are not written.
template <class T>
__device__ __forceinline__ typename Quad<T>::vec load_some(const T* p, int n)
{
    typename Quad<T>::vec v = {(T)0.0f, (T)0.0f, (T)0.0f, (T)0.0f};
    if (n > 0) v[0] = p[0];
    if (n > 1) v[1] = p[1];
    if (n > 2) v[2] = p[2];
    return v;
}

template <class T>
__device__ __forceinline__ void store_some(T* p, typename Quad<T>::vec v, int n)
{
    if (n > 0) p[0] = v[0];
    if (n > 1) p[1] = v[1];
    if (n > 2) p[2] = v[2];
}

// ---- AdamW ------------------------------------------------------------------

// A tensor, or 2^30 consecutive elements of a larger one, as a launch sees it.
struct Part32 {
    const void* g;
    void* p;
    void* m;
    void* v;
    float* master;
    uint32_t n;                            // at most 2^30
    // The factors of a step known to the host: 1 - lr_i wd and lr_i / (1 - beta1^t); of one read on the
    // device (t_dev): wd and the factor on the learning rate.
    float keep, step;
};
struct Part8 {
    const void* g;
    void* p;
    void* m;
    void* v;
    float* master;
    float* m_scale;
    float* v_scale;
    uint32_t n;
    float keep, step;
    uint32_t place;                        // tensor's index in the call's list * 2^10 + piece: the first
                                           // element is piece * 2^30
};
static_assert(sizeof(Part32) == 56 && sizeof(Part8) == 72, "the tables below are sized for these");
constexpr int64_t kPartElements = (int64_t)1 << 30;
constexpr int kPieceBits = 10;
constexpr int32_t kMostTensors = 1 << 22;

// Parts of one launch: the table rides in the kernel's arguments, which hold
// at most 4 KB, and a grid has fewer than 2^32 threads.
constexpr uint32_t kMostGroups = 1u << 23;

template <class Part, int MOST>
struct AdamwArgs {
    static constexpr int kMost = MOST;
    // The step's values from the host, or (t_dev) from the device's step and the schedule.
    float lr, beta1, beta2, eps;
    float root;                            // 1 / sqrt(1 - beta2^t) (t_dev: unset)
    uint32_t t;
    uint32_t k0, k1;                       // Philox key
    int32_t count;                         // parts
    uint32_t chunk;                        // elements per workgroup
    const float* gscale;
    const uint32_t* t_dev;
    ea_schedule_t sched;
    uint32_t first[MOST + 1];              // first workgroup of each part
    Part part[MOST];
};
using Adamw32Args = AdamwArgs<Part32, 64>;
using Adamw8Args = AdamwArgs<Part8, 52>;
static_assert(sizeof(Adamw32Args) <= 4096 && sizeof(Adamw8Args) <= 4096, "kernel arguments");

// The step's factors, formed in binary64 and rounded once, on the host or on the device alike.
__host__ __device__ inline double adamw_power(double b, uint32_t t)
{
    double r = 1.0;
    for (; t; t >>= 1) {
        if (t & 1) r = r * b;
        b = b * b;
    }
    return r;
}
__host__ __device__ inline float adamw_root(float beta2, uint32_t t)
{
    return (float)(1.0 / sqrt(1.0 - adamw_power((double)beta2, t)));
}
__host__ __device__ inline float adamw_step_size(double lri, float beta1, uint32_t t)
{
    return (float)(lri / (1.0 - adamw_power((double)beta1, t)));
}
__host__ __device__ inline float adamw_keep(double lri, float wd)
{
    return (float)(1.0 - lri * (double)wd);
}

// Elements per workgroup of a call of `total` elements, some with masters or none: what `first` counts in.
uint32_t adamw_chunk(const ea_adamw_t& c, int64_t total, bool masters);
hipError_t launch_adamw(const Adamw32Args& a, const ea_adamw_t& c, hipStream_t s);
hipError_t launch_adamw(const Adamw8Args& a, const ea_adamw_t& c, hipStream_t s);

// ---- gradient norm ------------------------------------------------------------

constexpr int kNormParts = 160;

struct NormArgs {
    int32_t count;                         // parts
    int64_t chunk;                         // elements per workgroup
    double* sums;                          // one per workgroup of this launch
    uint32_t first[kNormParts + 1];
    struct {
        const void* g;
        int64_t n;
    } part[kNormParts];
};
static_assert(sizeof(NormArgs) + 32 <= 4096, "kernel arguments");

// Gradients that one workgroup sums by itself, in one launch instead of two.  Issued from the host that
// takes 5.9 us against 8.5 to 9.3 while the GPU keeps up, which it does for up to 8 tensors (12: up to 11 us)
// and 131,072 elements in all (262,144: 9 to 14).  On the GPU alone (a graph) it takes 2 to 4 us against 3.4
// to 4.4 for up to 4 tensors and 65,536 elements, and up to 1.6 us more than two launches between 5 and 8
// tensors, 0.7 to 3.6 more at 131,072 elements: the limits keep what the host gains above what a graph loses.
constexpr int kSmallParts = 8;
constexpr int64_t kSmallTotal = 1 << 16;

int64_t norm_chunk(int64_t total);
hipError_t launch_norm(const NormArgs& a, int32_t grad_type, hipStream_t s);
bool norm_in_one(const NormArgs& a, int64_t total);
hipError_t launch_norm_small(const NormArgs& a, int32_t grad_type, float scale, float max_norm, float* norm,
                             float* gscale, hipStream_t s);
hipError_t launch_norm_finish(const double* part, int64_t parts, float scale, float max_norm, float* norm,
                              float* gscale, hipStream_t s);

// ---- embedding ----------------------------------------------------------------

hipError_t launch_embed_lookup(const ea_embed_t& c, const void* table, const void* ids, void* x, hipStream_t s);
int64_t embed_workspace_bytes(const ea_embed_t& c);
hipError_t launch_embed_grad(const ea_embed_t& c, const void* ids, const void* dx, void* dtable, bool accumulate,
                             void* workspace, hipStream_t s);

// t_dev[0] <- t_dev[0] + 1 (ea_kernels.hip).
hipError_t launch_advance(uint32_t* t_dev, hipStream_t s);

}  // namespace ea
