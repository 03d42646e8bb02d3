// Vectors of the three I/O types in float32 registers, and sums over wavefronts.  Device code only.
#ifndef GRKAN_VECTOR_H_
#define GRKAN_VECTOR_H_

#include <hip/hip_runtime.h>

namespace grkan {
namespace vec {

// VEC elements as they lie in memory, aligned to one element (the hardware takes vectors at any element; whole lines are the
// faster ones).
template <typename IO, int VEC> struct Raw {
    typedef IO type __attribute__((ext_vector_type(VEC), aligned(sizeof(IO))));
};
template <typename IO> struct Raw<IO, 1> {
    typedef IO type;
};

template <typename IO, int VEC> __device__ __forceinline__ typename Raw<IO, VEC>::type load(const IO *p)
{
    return *reinterpret_cast<const typename Raw<IO, VEC>::type *>(p);
}
template <typename IO, int VEC> __device__ __forceinline__ void widen(const typename Raw<IO, VEC>::type &r, float (&out)[VEC])
{
    if constexpr (VEC == 1)
        out[0] = (float)r;
    else
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            out[e] = (float)r[e];
}
// rounds to nearest even
template <typename IO, int VEC> __device__ __forceinline__ typename Raw<IO, VEC>::type narrow(const float (&in)[VEC])
{
    if constexpr (VEC == 1) {
        return (IO)in[0];
    } else {
        typedef float F __attribute__((ext_vector_type(VEC)));
        F f;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            f[e] = in[e];
        return __builtin_convertvector(f, typename Raw<IO, VEC>::type);
    }
}
template <typename IO, int VEC> __device__ __forceinline__ void store(IO *p, const typename Raw<IO, VEC>::type &r)
{
    *reinterpret_cast<typename Raw<IO, VEC>::type *>(p) = r;
}

// the same value in all lanes, in the same order every time
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
        v = o > v ? o : v;
    }
    return v;
}

} // namespace vec
} // namespace grkan
#endif // GRKAN_VECTOR_H_
