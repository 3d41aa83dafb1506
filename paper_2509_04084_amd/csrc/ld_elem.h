// Element types of the operators that take fp32, bf16 and fp16 arrays (LD_F32, LD_BF16, LD_F16): short vectors of them in
// memory, at any element's own alignment, and their values in 32 bits.
#pragma once

#include "ld_common.h"

static inline bool ld_known_type(int32_t dtype) { return dtype == LD_F32 || dtype == LD_BF16 || dtype == LD_F16; }
static inline int32_t ld_type_bytes(int32_t dtype) { return dtype == LD_F32 ? 4 : 2; }

// Calls f(integral_constant of the type) for a type known to be one of the three.
template <typename F>
static inline auto ld_with_type(int32_t dtype, F f) {
    if (dtype == LD_F32) return f(std::integral_constant<int, LD_F32>());
    if (dtype == LD_BF16) return f(std::integral_constant<int, LD_BF16>());
    return f(std::integral_constant<int, LD_F16>());
}

#ifdef __HIPCC__

template <int DT> struct LdElem { typedef float type; };
template <> struct LdElem<LD_BF16> { typedef __bf16 type; };
template <> struct LdElem<LD_F16> { typedef _Float16 type; };

// N elements side by side. Global memory takes vectors of up to 16 bytes at any address that its elements may have.
template <int DT, int N> struct LdVec {
    typedef typename LdElem<DT>::type elem;
    typedef elem type __attribute__((ext_vector_type(N), aligned(sizeof(elem))));
    typedef float wide __attribute__((ext_vector_type(N)));
    static __device__ __forceinline__ wide widen(type x) { return __builtin_convertvector(x, wide); }
    // rounded to nearest, ties to even
    static __device__ __forceinline__ type narrow(wide x) { return __builtin_convertvector(x, type); }
};

#endif  // __HIPCC__
