// What the elementwise kernels (adasum_checkpoint.cu, adasum_dropout.cu, adasum_fp8_pack.cu, adasum_residual_norm.cu)
// share: packed pairs of fp32 values, and vectors of eight elements as they lie in memory.
#pragma once

#include <type_traits>

#include "adasum_operators.cuh"

namespace adasum {

// ---- pairs of fp32 values ----------------------------------------------------------------------------
//
// With one instruction per value the checkpoint kernels were bound by instruction issue (30 instructions a value, 64 % of
// all issue slots at half the memory's speed); the packed forms do two values per instruction.

struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair pair_of(float a, float b)
{
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ Pair both(float a) { return pair_of(a, a); }
__device__ __forceinline__ float2 values_of(Pair p)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p.v));
    return f;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b)
{
    Pair c;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(c.v) : "l"(a.v), "l"(b.v));
    return c;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b)
{
    Pair c;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(c.v) : "l"(a.v), "l"(b.v));
    return c;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return d;
}
template <typename F>
__device__ __forceinline__ Pair each(Pair a, F f)
{
    const float2 v = values_of(a);
    return pair_of(f(v.x), f(v.y));
}

// ---- vectors of eight ----------------------------------------------------------------------------------

struct Eight {
    Pair p[4];
};

// A vector as it lies in memory: eight elements of T.
template <typename T>
struct Raw {
    uint4 w[sizeof(T) / 2];
};

// VEC: every row starts on 16 bytes and features is a multiple of 8, so each vector is either whole or only
// padding.  Otherwise the elements are taken one by one.
template <bool VEC, typename T>
__device__ __forceinline__ Raw<T> load_vector(const T* p, int count)
{
    Raw<T> raw;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i)
        raw.w[i] = make_uint4(0, 0, 0, 0);
    if constexpr (VEC) {
        if (count > 0) {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(T) / 2); ++i)
                raw.w[i] = reinterpret_cast<const uint4*>(p)[i];
        }
    } else {
        using Word = typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type;
        const Word* q = reinterpret_cast<const Word*>(p);
        uint32_t* w = reinterpret_cast<uint32_t*>(raw.w);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) {
                if constexpr (sizeof(T) == 4)
                    w[i] = q[i];
                else
                    w[i / 2] |= (uint32_t)q[i] << (16 * (i & 1));
            }
    }
    return raw;
}
template <typename T>
__device__ __forceinline__ Eight decode(const Raw<T>& raw)
{
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw.w);
    Eight x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (__is_same(T, float)) {
            x.p[i] = pair_of(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        } else if constexpr (__is_same(T, __half)) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x.p[i] = pair_of(f.x, f.y);
        } else {
            x.p[i] = pair_of(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        }
    }
    return x;
}
__device__ __forceinline__ void values_of(const Eight& x, float (&y)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = values_of(x.p[i]);
        y[2 * i] = f.x;
        y[2 * i + 1] = f.y;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_values(T* p, int count, const float (&y)[8])
{
    if constexpr (VEC) {
        if (count > 0)
            store_vector_from_float<8>(p, TypeCode<T>::value, 0, y);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count)
                store_from_float(p, TypeCode<T>::value, i, y[i]);
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_vector(T* p, int count, const Eight& x)
{
    float y[8];
    values_of(x, y);
    store_values<VEC>(p, count, y);
}

// Bits of the largest magnitude as an fp32 number; NaN or Inf (exponent 255) if there is one.
template <typename T>
__device__ __forceinline__ uint32_t largest(const Raw<T>& raw)
{
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw.w);
    if constexpr (__is_same(T, float)) {
        uint32_t top = 0;                       // as integers NaN > Inf > every number
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top = max(top, w[i] & 0x7fffffffu);
        return top;
    } else {
        using T2 = typename std::conditional<__is_same(T, __half), __half2, __nv_bfloat162>::type;
        auto half = [&](int i) { return __habs2(*reinterpret_cast<const T2*>(&w[i])); };
        const T2 m = __hmax2_nan(__hmax2_nan(half(0), half(1)), __hmax2_nan(half(2), half(3)));
        const float2 f = [&] {
            if constexpr (__is_same(T, __half))
                return __half22float2(m);
            else
                return __bfloat1622float2(m);
        }();
        return max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu);
    }
}

}  // namespace adasum
