// Loads and stores of several values at a time, for kernels that a type is a parameter of. Each
// translation unit has its own copy.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace flarepp {
namespace {
namespace vec {

template <int BYTES>
struct Word;
template <>
struct Word<16> { using t = uint4; };
template <>
struct Word<8> { using t = uint2; };
template <>
struct Word<4> { using t = uint32_t; };
template <>
struct Word<2> { using t = uint16_t; };

template <typename E, int N>
struct alignas(sizeof(E) * N) Pack {
    E v[N];
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float& d, float x) { d = x; }
__device__ __forceinline__ void narrow(__nv_bfloat16& d, float x) { d = __float2bfloat16_rn(x); }

template <typename E, int N>
__device__ __forceinline__ Pack<E, N> load(const E* p) {
    using W = typename Word<sizeof(E) * N>::t;
    const W w = *reinterpret_cast<const W*>(p);
    Pack<E, N> v;
    *reinterpret_cast<W*>(&v) = w;
    return v;
}
template <typename E, int N>
__device__ __forceinline__ void store(E* p, const Pack<E, N>& v) {
    using W = typename Word<sizeof(E) * N>::t;
    *reinterpret_cast<W*>(p) = *reinterpret_cast<const W*>(&v);
}

}  // namespace vec
}  // namespace
}  // namespace flarepp
