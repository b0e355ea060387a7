// smol_tokens_device.h -- what the token and attention kernels share: element
// types, loads and stores at element alignment, sums over a wave, division by a
// fixed divisor.
#ifndef SMOL_TOKENS_DEVICE_H
#define SMOL_TOKENS_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "smol_magic.h"

namespace smol {

typedef _Float16 f16;
typedef __bf16 bf16;

// N consecutive elements at the alignment of one: the device takes 16-byte
// global accesses at any element's address.
template <typename T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N)));
    typedef type loose __attribute__((aligned(sizeof(T))));
};
template <typename T, int N>
using vec = typename Vec<T, N>::type;

template <typename T, int N>
__device__ __forceinline__ vec<T, N> load(const T *p)
{
    typedef __attribute__((address_space(1))) const typename Vec<T, N>::loose In;
    return *(In *)p;
}

template <typename T, int N>
__device__ __forceinline__ void store(T *p, vec<T, N> v)
{
    typedef __attribute__((address_space(1))) typename Vec<T, N>::loose Out;
    *(Out *)p = v;
}

// The same for what is written once and not read again soon.
template <typename T, int N>
__device__ __forceinline__ void store_past(T *p, vec<T, N> v)
{
    typedef __attribute__((address_space(1))) typename Vec<T, N>::loose Out;
    __builtin_nontemporal_store(v, (Out *)p);
}

template <int N, typename T>
__device__ __forceinline__ vec<float, N> to_f32(vec<T, N> v)
{
    return __builtin_convertvector(v, vec<float, N>);
}

// To the nearest value of T, ties to even.
template <typename T, int N>
__device__ __forceinline__ vec<T, N> from_f32(vec<float, N> v)
{
    return __builtin_convertvector(v, vec<T, N>);
}

// Sum over the 64 lanes, the same value (and bits) in every lane: shifts
// within rows of 16 lanes, then row 0 into 1 and 2 into 3, then the lower
// half into the upper; lane 63 holds the sum.
__device__ __forceinline__ float wave_sum(float x)
{
#define SMOL_DPP_ADD(ctrl, rows)                                                                 \
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(                                 \
                                       0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, true))
    SMOL_DPP_ADD(0x111, 0xf);  // row_shr:1
    SMOL_DPP_ADD(0x112, 0xf);  // row_shr:2
    SMOL_DPP_ADD(0x114, 0xf);  // row_shr:4
    SMOL_DPP_ADD(0x118, 0xf);  // row_shr:8
    SMOL_DPP_ADD(0x142, 0xa);  // row_bcast:15 into rows 1 and 3
    SMOL_DPP_ADD(0x143, 0xc);  // row_bcast:31 into rows 2 and 3
#undef SMOL_DPP_ADD
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Division by a fixed divisor (smol_magic.h).
struct Divisor {
    uint32_t d, m, s;
};

inline Divisor make_divisor(uint32_t d)
{
    Divisor v;
    v.d = d;
    magic_divisor(d, &v.m, &v.s);
    return v;
}

__device__ __forceinline__ uint32_t divide(uint32_t n, const Divisor &v)
{
    return (uint32_t)((uint64_t)n * v.m >> v.s);
}

// Calls f with a value of the C++ type of an element type.
template <typename F>
auto with_type(int type, F f)
{
    return type == 0 ? f(float{}) : type == 1 ? f(f16{}) : f(bf16{});
}

inline int elem_size(int type) { return type == 0 ? 4 : 2; }

}  // namespace smol

#endif  // SMOL_TOKENS_DEVICE_H
