// Elements of 32 and 16 bits, widened to fp32 on the way in and rounded to nearest (ties to even) on the way out.
#pragma once
#include "common.hpp"

namespace bagua {

typedef uint16_t h4 __attribute__((ext_vector_type(4)));

template <int TYPE>
struct Elem {
    typedef uint16_t one;
    static __device__ __forceinline__ float widen(uint16_t x)
    {
        if (TYPE == BAGUA_BF16) return __uint_as_float(static_cast<uint32_t>(x) << 16);
        return static_cast<float>(__builtin_bit_cast(_Float16, x));
    }
    static __device__ __forceinline__ uint16_t narrow(float x)
    {
        if (TYPE == BAGUA_BF16) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
    }
};
template <>
struct Elem<BAGUA_F32> {
    typedef float one;
    static __device__ __forceinline__ float widen(float x) { return x; }
    static __device__ __forceinline__ float narrow(float x) { return x; }
};

inline size_t type_bytes(int type) { return type == BAGUA_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type >= BAGUA_F32 && type <= BAGUA_F16; }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace bagua
