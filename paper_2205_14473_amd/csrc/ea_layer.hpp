// ea_layer.hpp -- vectors of elements, reductions and launchers of the layers'
// operators (ea_layer.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ea_device.hpp"
#include "ea_layer.h"
#include "ea_train.hpp"

namespace ea {

// ---- vectors of N elements --------------------------------------------------

// N consecutive elements of type T at an address aligned to one element.
template <class T, int N>
struct VecOf {
    typedef T vec __attribute__((ext_vector_type(N)));
    typedef vec unaligned __attribute__((aligned(sizeof(T))));
};
template <class T>
struct VecOf<T, 1> {
    typedef T vec;
    typedef T unaligned;
};
template <class T, int N>
using Vec = typename VecOf<T, N>::vec;

template <int N, class T>
__device__ __forceinline__ Vec<T, N> load_vec(const T* p)
{
    return *(const typename VecOf<T, N>::unaligned*)p;
}

// ONCE: past the caches.
template <int N, bool ONCE = false, class T>
__device__ __forceinline__ void store_vec(T* p, Vec<T, N> v)
{
    typedef typename VecOf<T, N>::unaligned At;
    if (ONCE)
        __builtin_nontemporal_store(v, (At*)p);
    else
        *(At*)p = v;
}

// Arrays from this size on are written past the caches: little of them would be left in the last one when the next call
// reads them, and what is there makes way.  (Norm, recurrence, dropout, loss and their gradients in a row, arrays of
// 16 MiB each: 131 us, and 138 past the caches; of 64 MiB: 333 and 329; of 256 MiB: 1,091 and 1,070.  Loads past them,
// too, gain where an array comes from memory, and lose more where the call before left it: 333 and 348 at 64 MiB.)
constexpr int64_t kOnceBytes = (int64_t)64 << 20;

inline bool past_caches(int64_t elements, int32_t type)
{
    return elements >= kOnceBytes / (type == EA_F32 ? 4 : 2);
}

template <class F>
hipError_t with_bool(bool on, F&& f)
{
    return on ? f(std::true_type{}) : f(std::false_type{});
}

// Element k of a vector, also of one of a single element.
template <int N, class T>
__device__ __forceinline__ T element(const Vec<T, N>& v, int k)
{
    if constexpr (N == 1)
        return v;
    else
        return v[k];
}

template <int N, class T>
__device__ __forceinline__ void set_element(Vec<T, N>& v, int k, T x)
{
    if constexpr (N == 1)
        v = x;
    else
        v[k] = x;
}

// The first `n` elements; the rest read as `rest`, and are not written.  All loads are made at once, the rest's from
// the first element: a branch around each would make a row wait N times for memory.
template <int N, class T>
__device__ __forceinline__ Vec<T, N> load_part(const T* p, int n, float rest = 0.0f)
{
    Vec<T, N> v;
#pragma unroll
    for (int k = 0; k < N; ++k) set_element<N, T>(v, k, (T)rest);
    if (n > 0) {
        T x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = p[k < n ? k : 0];
#pragma unroll
        for (int k = 0; k < N; ++k) set_element<N, T>(v, k, k < n ? x[k] : (T)rest);
    }
    return v;
}

template <int N, class T>
__device__ __forceinline__ void store_part(T* p, Vec<T, N> v, int n)
{
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < n) p[k] = element<N, T>(v, k);
}

template <int N, class T>
__device__ __forceinline__ void widen_to(float* x, const Vec<T, N>& v)
{
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = (float)element<N, T>(v, k);
}

template <int N, class T>
__device__ __forceinline__ Vec<T, N> narrow_from(const float* x)
{
    Vec<T, N> v;
#pragma unroll
    for (int k = 0; k < N; ++k) set_element<N, T>(v, k, (T)x[k]);
    return v;
}

// One element of a tensor whose type is known when it runs only, for what is read once per column.
__device__ __forceinline__ float element_at(const void* p, int32_t type, int64_t i)
{
    if (type == EA_F32) return ((const float*)p)[i];
    if (type == EA_BF16) return (float)((const bf16*)p)[i];
    return (float)((const f16*)p)[i];
}

__device__ __forceinline__ void set_element_at(void* p, int32_t type, int64_t i, float x)
{
    if (type == EA_F32)
        ((float*)p)[i] = x;
    else if (type == EA_BF16)
        ((bf16*)p)[i] = (bf16)x;
    else
        ((f16*)p)[i] = (f16)x;
}

// ---- reductions ---------------------------------------------------------------

// All 64 lanes end with the same bits.
__device__ __forceinline__ float wave_sum(float v)
{
    v = v + __uint_as_float(dpp<kDppXor1>(__float_as_uint(v)));
    v = v + __uint_as_float(dpp<kDppXor2>(__float_as_uint(v)));
    v = v + __uint_as_float(dpp<kDppHalfMirror>(__float_as_uint(v)));
    v = v + __uint_as_float(dpp<kDppRowMirror>(__float_as_uint(v)));
    uint32_t a, b;
    row_swap16(__float_as_uint(v), a, b);
    v = __uint_as_float(a) + __uint_as_float(b);
    row_swap32(__float_as_uint(v), a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}

// ---- types at run time ----------------------------------------------------------

// f with a value of the element type: f(float{}), f(bf16{}) or f(f16{}).
template <class F>
hipError_t with_type(int32_t type, F&& f)
{
    if (type == EA_F32) return f(float{});
    if (type == EA_BF16) return f(bf16{});
    return f(f16{});
}

// ---- launchers ------------------------------------------------------------------

hipError_t launch_layer_norm(const ea_layer_norm_t& c, const void* x, const void* weight, const void* bias, void* y,
                             float* mean, float* rstd, hipStream_t s);
int64_t layer_norm_workspace_bytes(const ea_layer_norm_t& c);
hipError_t launch_layer_norm_grad(const ea_layer_norm_t& c, const void* x, const void* dy, const void* weight,
                                  const float* mean, const float* rstd, const void* add, void* dx, void* dweight,
                                  void* dbias, bool accumulate, void* workspace, hipStream_t s);

// residual is NULL for the gradient, whose dy takes x's place.
hipError_t launch_dropout(const ea_dropout_t& c, bool backward, uint32_t t, const uint32_t* t_dev, const void* in,
                          const void* residual, void* out, hipStream_t s);

int64_t recurrence_workspace_bytes(const ea_recurrence_t& c);
hipError_t launch_recurrence(const ea_recurrence_t& c, const void* g, const void* x, const float* h0,
                             const int32_t* lengths, void* y, float* states, float* h_last, void* workspace,
                             hipStream_t s);
hipError_t launch_recurrence_grad(const ea_recurrence_t& c, const void* g, const void* x, const float* states,
                                  const int32_t* lengths, const void* dy, const float* dh_last, void* dg, void* dx,
                                  float* dh0, void* workspace, hipStream_t s);

int64_t token_loss_workspace_bytes(const ea_token_loss_t& c);
hipError_t launch_token_loss(const ea_token_loss_t& c, const void* logits, const void* targets, float* loss,
                             float* total, int32_t* count, void* dlogits, void* workspace, hipStream_t s);

}  // namespace ea
