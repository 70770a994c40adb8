// Elements of 32 and 16 bits, widened to fp32 on the way in and rounded to nearest (ties to even) on the way out.  Vectors are
// declared with the alignment of one element: the hardware takes a wide access at any address.
#pragma once
#include "common.hpp"

namespace bagua {

typedef uint16_t h4 __attribute__((ext_vector_type(4)));
typedef uint16_t h4e __attribute__((ext_vector_type(4), aligned(2)));

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
    static __device__ __forceinline__ f4 load(const uint16_t* p)
    {
        const h4e v = __builtin_nontemporal_load(reinterpret_cast<const h4e*>(p));
        return f4{widen(v.x), widen(v.y), widen(v.z), widen(v.w)};
    }
    static __device__ __forceinline__ void store(uint16_t* p, f4 v)
    {
        __builtin_nontemporal_store(h4e{narrow(v.x), narrow(v.y), narrow(v.z), narrow(v.w)}, reinterpret_cast<h4e*>(p));
    }
};
template <>
struct Elem<BAGUA_F32> {
    typedef float one;
    static __device__ __forceinline__ float widen(float x) { return x; }
    static __device__ __forceinline__ float narrow(float x) { return x; }
    static __device__ __forceinline__ f4 load(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f4u*>(p)); }
    static __device__ __forceinline__ void store(float* p, f4 v) { __builtin_nontemporal_store(static_cast<f4u>(v), reinterpret_cast<f4u*>(p)); }
};

inline size_t type_bytes(int type) { return type == BAGUA_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type >= BAGUA_F32 && type <= BAGUA_F16; }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace bagua
