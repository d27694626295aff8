// ea_layer_norm.hpp -- what layer norm and its gradient share: a row's vectors,
// sums over the waves of a row, and how many waves hold one.
#pragma once

#include <type_traits>

#include "ea_layer.hpp"

namespace ea {

namespace norm {

constexpr int kHeldColumns = 16;                       // a lane's, at most
constexpr int kLongBlock = 1024;                       // threads of a row that is not held

// Elements of a vector: 16 bytes of the narrower type, or four where rows are no whole number of those (TAIL).
template <class X, class Y, bool TAIL>
constexpr int vec_of()
{
    return !TAIL && sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
}

template <class X, class Y, bool TAIL>
constexpr int kVec = vec_of<X, Y, TAIL>();

// A vector moved down by some of its elements, zeros behind.
template <int V, class T>
__device__ __forceinline__ Vec<T, V> moved_down(Vec<T, V> v, int by)
{
    const int bits = by * 8 * (int)sizeof(T), rest = bits & 63;
    if constexpr (sizeof(v) == 16) {
        typedef uint64_t Two __attribute__((ext_vector_type(2)));
        const Two w = __builtin_bit_cast(Two, v);
        const uint64_t low = bits < 64 ? w[0] : w[1], high = bits < 64 ? w[1] : 0;
        const Two moved = {(low >> rest) | (rest ? high << (64 - rest) : 0), high >> rest};
        return __builtin_bit_cast(Vec<T, V>, moved);
    } else {
        return __builtin_bit_cast(Vec<T, V>, __builtin_bit_cast(uint64_t, v) >> rest);
    }
}

constexpr int kTail = 1, kTiny = 2;

// The tail of a lane's vector k of K.
template <bool TAIL, int WAVES, int K>
__device__ __forceinline__ constexpr int tail_of(int k)
{
    return !TAIL || k < K - 1 ? 0 : WAVES * K == 1 ? kTiny : kTail;
}

// The row's vector at column `at`, zeros behind its end.  tail: it may cross the end; it is then the row's last whole
// one, moved down, so that a vector is one load and nothing outside the row is read (kTiny: the row may be shorter than
// one).  (Elements one by one for rows of no whole number of vectors: 65,536 x 1,001 bfloat16 135 us and 378 the
// gradient, this way 47 and 106.)
template <int V, class T>
__device__ __forceinline__ Vec<T, V> row_vec(const T* row, int at, int dim, int tail)
{
    Vec<T, V> v = {};
    if (tail == kTiny && dim < V) {
        v = load_part<V>(row + at, dim - at);
    } else if (at < dim) {
        const int from = !tail || at < dim - V ? at : dim - V;
        v = *(const typename VecOf<T, V>::unaligned*)((const char*)row + (uint32_t)from * (uint32_t)sizeof(T));
        if (tail) v = moved_down<V, T>(v, at - from);
    }
    return v;
}

template <int V, class T>
__device__ __forceinline__ void load_row(float* x, const T* row, int at, int dim, int tail)
{
    if constexpr (sizeof(T) * V > 16) {
        load_row<V / 2>(x, row, at, dim, tail);
        load_row<V / 2>(x + V / 2, row, at + V / 2, dim, tail);
    } else {
        widen_to<V, T>(x, row_vec<V>(row, at, dim, tail));
    }
}

template <int V, bool ONCE = false, class T>
__device__ __forceinline__ void store_row(T* row, int at, const float* x, int dim, bool tail)
{
    T* to = (T*)((char*)row + (uint32_t)at * (uint32_t)sizeof(T));
    if (at < dim && (!tail || at + V <= dim))
        store_vec<V, ONCE>(to, narrow_from<V, T>(x));
    else if (tail && at < dim)
        store_part<V>(to, narrow_from<V, T>(x), dim - at);
}

// weight or bias, or what stands for it where there is none
template <int V>
__device__ __forceinline__ void load_weights(float* x, const void* w, int32_t type, int at, int dim, float none,
                                             int tail)
{
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = none;
    if (!w) return;
    if (type == EA_F32)
        load_row<V>(x, (const float*)w, at, dim, tail);
    else if (type == EA_BF16)
        load_row<V>(x, (const bf16*)w, at, dim, tail);
    else
        load_row<V>(x, (const f16*)w, at, dim, tail);
}

// Sums of one or two values over the waves of a row; every thread gets them.
template <int WAVES>
__device__ __forceinline__ void row_sums(float& a, float& b, float2* lds)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if (WAVES == 1) return;
    const int wave = wave_id();
    if (lane_id() == 0) lds[wave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
        a = a + lds[k].x;
        b = b + lds[k].y;
    }
    __syncthreads();
}

// sum / n, where each is 1 / n rounded: what the product leaves of the sum comes out of one operation and corrects it to
// the nearest.  (Of an infinite sum it leaves NaN, and there is nothing to correct.)
// (131,072 x 256 bfloat16, mean and variance by divisions of ten operations each: 31.4 us; without: 28.0.)
__device__ __forceinline__ float quotient(float sum, float n, float each)
{
    const float q = sum * each, left = __builtin_fmaf(-q, n, sum);
    return left == left ? __builtin_fmaf(left, each, q) : q;
}

// Waves of a row and vectors a lane holds of it (0 waves: the row is not held), the fewest that hold it, so that only a
// lane's last vector may cross the row's end; whether one does.
struct Shape {
    int waves, k;
    bool tail;
};

inline Shape shape_of(const ea_layer_norm_t& c)
{
    const int whole = c.x_type != EA_F32 && c.y_type != EA_F32 ? 8 : 4;
    const bool tail = c.dim % whole != 0;
    const int v = tail ? 4 : whole;
    for (int waves = 1; waves <= 16; waves *= 4)
        for (int k = 1; k * v <= kHeldColumns; ++k)
            if (c.dim <= (int64_t)waves * kWave * k * v) return {waves, k, tail};
    return {0, 0, tail};
}

// f with the tail, the waves and the vectors a lane as constants.
template <int V, class F>
hipError_t with_shape(Shape s, F&& f)
{
#define EA_SHAPE(T, W, K)                           \
    if (s.tail == T && s.waves == W && s.k == K)    \
    return f(std::integral_constant<bool, T>{}, std::integral_constant<int, W>{}, std::integral_constant<int, K>{})
#define EA_WAVES(T, K)   \
    EA_SHAPE(T, 1, K);   \
    EA_SHAPE(T, 4, K);   \
    EA_SHAPE(T, 16, K)
    EA_WAVES(false, 1);
    EA_WAVES(false, 2);
    if constexpr (V == 4) {
        EA_WAVES(false, 3);
        EA_WAVES(false, 4);
    }
    EA_WAVES(true, 1);
    EA_WAVES(true, 2);
    EA_WAVES(true, 3);
    EA_WAVES(true, 4);
#undef EA_WAVES
#undef EA_SHAPE
    return hipErrorInvalidValue;
}

inline int64_t at_most(int64_t n, int64_t most)
{
    return n < most ? n : most;
}

}  // namespace norm
}  // namespace ea
