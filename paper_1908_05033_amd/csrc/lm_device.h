// Device-side helpers of the language-model kernels (gfx950 only).
#pragma once
#include "lm_kernels.h"

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

// N elements that lie side by side in memory, at any alignment of the element: loads and stores of a row whose length
// is odd are still one instruction (global memory takes dword accesses at any address).
template <class E, int N>
struct __attribute__((packed)) Side {
    E at[N];
};

template <class E, int N>
__device__ __forceinline__ Side<E, N> load_side(const E *p)
{
    return *reinterpret_cast<const Side<E, N> *>(p);
}
template <class E, int N>
__device__ __forceinline__ void store_side(E *p, const Side<E, N> &v)
{
    *reinterpret_cast<Side<E, N> *>(p) = v;
}

template <int T>
struct Element;
template <>
struct Element<DSQ_T_F32> {
    typedef float type;
};
template <>
struct Element<DSQ_T_F16> {
    typedef _Float16 type;
};
template <>
struct Element<DSQ_T_BF16> {
    typedef __bf16 type;
};
template <>
struct Element<DSQ_T_I8> {
    typedef int8_t type;
};
