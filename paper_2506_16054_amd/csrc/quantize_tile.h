// What the kernels around the block quantizer share (paper Sec. 4.3 (1)): reading and writing eight channels of a token.
#pragma once

#include "common.h"

namespace paro {

template <typename T>
__device__ inline void load8(const T* p, float (&x)[8]);

template <>
__device__ inline void load8<float>(const float* p, float (&x)[8]) {
    const float4 a = ((const float4*)p)[0];
    const float4 b = ((const float4*)p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

template <>
__device__ inline void load8<uint16_t>(const uint16_t* p, float (&x)[8]) {  // bf16 bit patterns
    // the input is read exactly once: a non-temporal load keeps it from displacing the codes in the caches
    // (-3 % on the one-grid quantizer; the same hint on the stores of the codes, which the attention kernel reads
    // next, gains nothing)
    typedef unsigned v4u __attribute__((ext_vector_type(4)));
    const v4u a = __builtin_nontemporal_load((const v4u*)p);
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// eight values that load8 read, as they were
__device__ inline void store8(float* p, const float (&x)[8]) {
    ((float4*)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4*)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ inline void store8(uint16_t* p, const float (&x)[8]) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ inline unsigned f32_to_bf16_bits(float f) {  // round to nearest even
    const unsigned u = __float_as_uint(f);
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

__device__ inline float wave_max(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

}  // namespace paro
