// Elements of 32 and 16 bits: loads into and stores from fp32, four at a time and one by one, at any alignment of the element type.
#pragma once

#include <type_traits>

#include "atomo_internal.h"

namespace atomo {

// (four elements from an address that is a multiple of one element's size: one instruction all the same)
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint16_t u16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

inline int type_bytes(int type) { return type == ATOMO_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == ATOMO_F32 || type == ATOMO_BF16 || type == ATOMO_F16; }

// A conversion from fp32 rounds to the nearest, ties to even: what is stored is what was formed in fp32, once.
template <int TYPE> struct Element;
template <> struct Element<ATOMO_F32> {
    typedef float Stored;
    typedef f32x4_any Stored4;
    __device__ static float up(Stored x) { return x; }
    __device__ static Stored down(float x) { return x; }
};
template <> struct Element<ATOMO_BF16> {
    typedef uint16_t Stored;
    typedef u16x4_any Stored4;
    __device__ static float up(Stored x) { return __uint_as_float((uint32_t)x << 16); }
    __device__ static Stored down(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <> struct Element<ATOMO_F16> {
    typedef uint16_t Stored;
    typedef u16x4_any Stored4;
    __device__ static float up(Stored x) { return (float)__builtin_bit_cast(_Float16, x); }
    __device__ static Stored down(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};

// ONCE: what a kernel reads or writes once and the caches need not keep.
template <int TYPE, bool ONCE = false>
__device__ inline f32x4 load4(const void* base, long long i)
{
    const auto at = (const typename Element<TYPE>::Stored4*)((const typename Element<TYPE>::Stored*)base + i);
    const auto s = ONCE ? __builtin_nontemporal_load(at) : *at;
    return f32x4{Element<TYPE>::up(s[0]), Element<TYPE>::up(s[1]), Element<TYPE>::up(s[2]), Element<TYPE>::up(s[3])};
}

template <int TYPE, bool ONCE = false>
__device__ inline void store4(void* base, long long i, f32x4 x)
{
    typename Element<TYPE>::Stored4 s;
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = Element<TYPE>::down(x[k]);
    const auto at = (typename Element<TYPE>::Stored4*)((typename Element<TYPE>::Stored*)base + i);
    if constexpr (ONCE) __builtin_nontemporal_store(s, at);
    else *at = s;
}

template <int TYPE>
__device__ inline float load1(const void* base, long long i)
{
    return Element<TYPE>::up(((const typename Element<TYPE>::Stored*)base)[i]);
}

template <int TYPE>
__device__ inline void store1(void* base, long long i, float x)
{
    ((typename Element<TYPE>::Stored*)base)[i] = Element<TYPE>::down(x);
}

// Calls f with an integral constant for a type that is only known at run time (known_type has been asked).
template <typename F>
inline auto with_type(int type, F&& f)
{
    if (type == ATOMO_BF16) return f(std::integral_constant<int, ATOMO_BF16>());
    if (type == ATOMO_F16) return f(std::integral_constant<int, ATOMO_F16>());
    return f(std::integral_constant<int, ATOMO_F32>());
}

}  // namespace atomo
